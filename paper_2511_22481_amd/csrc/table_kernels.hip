// Block tables and slot maps on the device.
//
// One step lets request b grow from L_b to L_b + n_b tokens.  It then has ceil((L_b + n_b) / 128) pages, and takes the
// ones it lacks from the top of the pool's stack of free pages, in the order of the requests: with N_b the running sum
// of the pages that requests up to b lack, page k of request b is free[count - 1 - (N_b - need_b) - k].  Everything
// follows from two running sums over the batch (tokens and pages), so no entry waits for another request's.
//
// What bounds it: a launch and a chain of dependent loads.  64 requests of a token 2.4 us, 256 of which 32 bring up to 512 tokens 4.5, 1500 requests'
// prompts (25000 slots) 5.9.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "gqa.h"

namespace omniattn {
namespace {

constexpr int kThreads = 1024;  // at most; also the requests whose sums are held in LDS at a time
constexpr uint32_t kMost = 0x7fffffffu;

// Sums stop at the largest int32: a batch whose lengths are nonsense gets no pages, but nothing wraps.
__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) { return min(a + b, kMost); }

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + kPage - 1) / kPage); }

// Running sum over a wave, or (rows of 16 only) over each 16 lanes.
template <bool WAVE>
__device__ __forceinline__ uint32_t sum_up_to(uint32_t x) {
#define OMNIATTN_ADD(ctrl, rows) x = sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, true))
  OMNIATTN_ADD(0x111, 0xf);  // from the lane one, two, four, eight before, in rows of 16
  OMNIATTN_ADD(0x112, 0xf);
  OMNIATTN_ADD(0x114, 0xf);
  OMNIATTN_ADD(0x118, 0xf);
  if constexpr (WAVE) {
    OMNIATTN_ADD(0x142, 0xa);  // a row's last lane to the row behind it
    OMNIATTN_ADD(0x143, 0xc);  // lane 31 to the upper half
  }
#undef OMNIATTN_ADD
  return x;
}

// Sum over the work group's threads before this one.  `tot`: one word per wave, to be left alone until the caller's next barrier.  One barrier.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t* tot) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / 64;
  x = sum_up_to<true>(x);
  if (lane == 63) tot[wave] = x;
  __syncthreads();
  const uint32_t ends = sum_up_to<false>(lane < waves ? tot[lane] : 0);  // (up to 16 waves)
  const uint32_t before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)ends, wave - 1) : 0;
  x = __shfl_up(x, 1);
  return lane ? sat(x, before) : before;
}

// First index whose running sum is above i (n entries, the last one is).
__device__ __forceinline__ int owner(const uint32_t* ends, int n, uint32_t i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (ends[mid] > i) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// WHAT: 1 table, first tokens and slots; 2 lengths and the stack's height; 3 both.  Every work group sums over the whole
// batch by itself (its lengths are a few KB in L2) and writes its share of the slots and table entries, so one launch
// does it and no group waits for another.  Only where the new lengths replace the old ones in place must the writing of
// them come behind all reading: a launch of its own, or the only work group.  PER: neighbouring requests to a thread; batches of
// more than PER work groups' threads take several turns, one behind the other.
template <int WHAT, int PER>
__global__ __launch_bounds__(kThreads) void extend_kernel(TableParams p) {
  constexpr int kMany = PER * kThreads;
  __shared__ uint32_t tot[2][kThreads / 64];
  __shared__ uint32_t token_end[kMany], page_end[kMany];
  __shared__ int had[kMany], len[kMany];  // had: -1 where the request is refused
  const int tid = threadIdx.x, threads = blockDim.x;
  const bool first_group = blockIdx.x == 0;
  const int count = *p.free_count;
  const uint32_t free = (uint32_t)max(count, 0);
  uint32_t tokens = 0, pages = 0, used = 0;  // sums over the chunks before; pages granted
  for (int b0 = 0; b0 < p.batch; b0 += PER * threads) {
    int L[PER], n[PER], start_page[PER];
    uint32_t sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int b = b0 + tid * PER + j;
      L[j] = b < p.batch ? p.seq_lens[b] : 0;
      n[j] = b < p.batch ? p.new_lens[b] : 0;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int b = b0 + tid * PER + j;
      if constexpr (PER == 1) start_page[j] = b < p.batch && L[j] >= 0 && L[j] / kPage < p.max_pages && n[j] > 0 ? p.page_table[b * p.stride + L[j] / kPage] : 0;
      sum = sat(sum, (uint32_t)max(n[j], 0));
    }
    // (a sum that has stopped is no request's first token: refused below)
    uint32_t t_end[PER], p_end[PER], need[PER];
    bool fine[PER];
    uint32_t run = sat(tokens, sum_before(sum, tot[0]));
    sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool mine = b0 + tid * PER + j < p.batch;
      const int64_t after = (int64_t)L[j] + n[j];
      t_end[j] = run = sat(run, (uint32_t)max(n[j], 0));
      fine[j] = mine && L[j] >= 0 && n[j] >= 0 && pages_of(after) <= p.max_pages && t_end[j] <= (uint32_t)p.max_tokens && t_end[j] < kMost;
      need[j] = fine[j] ? (uint32_t)(pages_of(after) - pages_of(L[j])) : 0;
      sum = sat(sum, need[j]);
    }
    run = sat(pages, sum_before(sum, tot[1]));
    bool more = false;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int at = tid * PER + j, b = b0 + at;
      p_end[j] = run = sat(run, need[j]);
      fine[j] = fine[j] && (need[j] == 0 || p_end[j] <= free);
      if (first_group && b < p.batch) {
        if constexpr (WHAT & 2) p.seq_lens_out[b] = fine[j] ? L[j] + n[j] : L[j];
        if constexpr (WHAT & 1) {
          p.q_start[b + 1] = (int)t_end[j];
          if (b == 0) p.q_start[0] = 0;
        }
      }
      token_end[at] = t_end[j];
      page_end[at] = p_end[j];
      had[at] = fine[j] ? pages_of(L[j]) : -1;
      len[at] = L[j];
      more = more || n[j] > 1;
    }
    // (whether all of the chunk's requests bring one token at most: a decode step)
    const bool chunky = __syncthreads_or(more) || PER > 1;
    const int last = min(PER * threads, p.batch - b0) - 1;
    if constexpr (WHAT & 1) {
      if (!chunky) {
        const int b = b0 + tid;
        if (first_group && b < p.batch && n[0] == 1 && t_end[0] <= (uint32_t)p.max_tokens) {
          int slot = -1;
          if (fine[0]) {
            const int page = need[0] ? p.free_pages[free - p_end[0]] : start_page[0];
            if (need[0]) p.page_table[b * p.stride + pages_of(L[0])] = page;
            slot = page * kPage + L[0] % kPage;
          }
          p.slot_map[t_end[0] - 1] = slot;
        }
      } else {
        const uint32_t step = gridDim.x * threads, at = blockIdx.x * threads + tid;
        // table entries (granted requests come before the first that the stack has no pages for)
        const uint32_t page_stop = min(page_end[last], free);
        for (uint32_t k = pages + at; k < page_stop; k += step) {
          const int o = owner(page_end, last + 1, k);
          const uint32_t begin = o ? page_end[o - 1] : pages;
          if (had[o] >= 0 && page_end[o] <= free) p.page_table[(b0 + o) * p.stride + had[o] + (int)(k - begin)] = p.free_pages[free - 1 - k];
        }
        const uint32_t token_stop = min(token_end[last], (uint32_t)p.max_tokens);
        for (uint32_t i = tokens + at; i < token_stop; i += step) {
          const int o = owner(token_end, last + 1, i);
          int slot = -1;
          if (had[o] >= 0) {
            const int pos = len[o] + (int)(i - (o ? token_end[o - 1] : tokens));
            const int lp = pos / kPage;
            // (pages taken in this call: from the stack, not from the table that other work groups are writing)
            const int page = lp < had[o] ? p.page_table[(b0 + o) * p.stride + lp]
                                         : p.free_pages[free - 1 - ((o ? page_end[o - 1] : pages) + (uint32_t)(lp - had[o]))];
            slot = page * kPage + pos % kPage;
          }
          p.slot_map[i] = slot;
        }
      }
    }
    if constexpr (WHAT & 2) {
      // pages granted up to here: the largest sum that the stack covers, of a request that needed any
      if (first_group) {
        for (int o = tid; o <= last; o += threads) {
          const uint32_t begin = o ? page_end[o - 1] : pages;
          if (had[o] >= 0 && page_end[o] > begin && page_end[o] <= free) used = max(used, page_end[o]);
        }
      }
    }
    tokens = token_end[last];
    pages = page_end[last];
    if (b0 + PER * threads < p.batch) __syncthreads();  // the sums are read before the next chunk's replace them
  }
  if constexpr (WHAT & 1) {
    for (uint32_t i = tokens + blockIdx.x * threads + tid; i < (uint32_t)p.max_tokens; i += gridDim.x * threads) p.slot_map[i] = -1;
  }
  if constexpr (WHAT & 2) {
    if (first_group) {
      for (int d = 1; d < 64; d *= 2) used = max(used, (uint32_t)__shfl_xor(used, d));
      if ((tid & 63) == 0) tot[0][tid >> 6] = used;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < threads / 64; ++w) used = max(used, tot[0][w]);
        *p.free_count_out = count - (int)used;
      }
    }
  }
}

// The pages of finished requests go back on the stack, in the order of the requests.  One work group: a step finishes
// few requests, and the stack's height and the lengths change in place.
__global__ __launch_bounds__(kThreads) void release_kernel(ReleaseParams p) {
  __shared__ uint32_t tot[kThreads / 64];
  __shared__ uint32_t page_end[kThreads];
  const int tid = threadIdx.x;
  const int count = max(*p.free_count, 0);
  uint32_t pages = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    const int b = b0 + tid;
    const bool gone = b < p.batch && p.done[b] != 0;
    const int L = gone ? p.seq_lens[b] : 0;
    const uint32_t many = (uint32_t)min(pages_of(max(L, 0)), p.max_pages), end = sat(sat(pages, sum_before(many, tot)), many);
    page_end[tid] = end;
    if (gone) p.seq_lens[b] = 0;
    __syncthreads();
    const uint32_t stop = page_end[kThreads - 1];
    for (uint32_t k = pages + tid; k < stop; k += kThreads) {
      const int o = owner(page_end, kThreads, k);
      // (a stack that is already full takes no more: pages released twice)
      if ((int64_t)count + k < p.num_pages) p.free_pages[count + k] = p.page_table[(b0 + o) * p.stride + (int)(k - (o ? page_end[o - 1] : pages))];
    }
    pages = stop;
    __syncthreads();
  }
  if (tid == 0) *p.free_count = (int)min((int64_t)count + pages, p.num_pages);
}

}  // namespace

hipError_t launch_table_extend(const TableParams& p, hipStream_t stream) {
  // A thread to a request, or to two where there are more than threads (1500 requests: 11.7 us in two turns), and at least 256; as many work
  // groups as there are slots for them (256 requests with chunks: 6.8 us with 1024 threads each).
  const bool pairs = p.batch > kThreads;
  const int want = std::max(pairs ? (p.batch + 1) / 2 : p.batch, std::min(p.max_tokens, 256));
  const int threads = std::min(kThreads, (want + 63) / 64 * 64);
  const int groups = std::max(1, std::min(256, (p.max_tokens + threads - 1) / threads));
  const bool in_place = p.seq_lens_out == p.seq_lens || p.free_count_out == p.free_count;
  auto launch = [&](auto what, int grid) {
    constexpr int kWhat = decltype(what)::value;
    if (pairs) hipLaunchKernelGGL((extend_kernel<kWhat, 2>), dim3(grid), dim3(threads), 0, stream, p);
    else hipLaunchKernelGGL((extend_kernel<kWhat, 1>), dim3(grid), dim3(threads), 0, stream, p);
    return hipGetLastError();
  };
  if (!in_place || groups == 1) return launch(std::integral_constant<int, 3>{}, groups);
  const hipError_t e = launch(std::integral_constant<int, 1>{}, groups);
  return e != hipSuccess ? e : launch(std::integral_constant<int, 2>{}, 1);
}

hipError_t launch_table_release(const ReleaseParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace omniattn
