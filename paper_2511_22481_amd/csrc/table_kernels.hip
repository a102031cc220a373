// Block tables and slot maps on the device.
//
// One step lets request b grow from L_b to L_b + n_b tokens.  It then has ceil((L_b + n_b) / 128) pages, and takes the
// ones it lacks from the top of the pool's stack of free pages, in the order of the requests: with N_b the running sum
// of the pages that requests up to b lack, page k of request b is free[count - 1 - (N_b - need_b) - k].  Everything
// follows from two running sums over the batch (tokens and pages), so no entry waits for another request's.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gqa.h"

namespace omniattn {
namespace {

constexpr int kThreads = 1024;  // at most; also the requests whose sums are held in LDS at a time
constexpr uint32_t kMost = 0x7fffffffu;

// Sums stop at the largest int32: a batch whose lengths are nonsense gets no pages, but nothing wraps.
__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) { return min(a + b, kMost); }

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + kPage - 1) / kPage); }

// Inclusive running sum over the work group's threads.  `tot`: one word per wave; two barriers.
__device__ __forceinline__ uint32_t group_sum(uint32_t x, uint32_t* tot) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x = sat(x, y);
  }
  __syncthreads();
  if (lane == 63) tot[wave] = x;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before = sat(before, tot[w]);
  return sat(x, before);
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
// them come behind all reading: a launch of its own, or the only work group.
template <int WHAT>
__global__ __launch_bounds__(kThreads) void extend_kernel(TableParams p) {
  __shared__ uint32_t tot[kThreads / 64];
  __shared__ uint32_t token_end[kThreads], page_end[kThreads];
  __shared__ int had[kThreads], len[kThreads];  // had: -1 where the request is refused
  const int tid = threadIdx.x, threads = blockDim.x;
  const bool first_group = blockIdx.x == 0;
  const int count = *p.free_count;
  const uint32_t free = (uint32_t)max(count, 0);
  uint32_t tokens = 0, pages = 0, used = 0;  // sums over the chunks before; pages granted
  for (int b0 = 0; b0 < p.batch; b0 += threads) {
    const int b = b0 + tid;
    const bool mine = b < p.batch;
    const int L = mine ? p.seq_lens[b] : 0, n = mine ? p.new_lens[b] : 0;
    const int start_page = mine && L >= 0 && L / kPage < p.max_pages && n > 0 ? p.page_table[b * p.stride + L / kPage] : 0;
    const uint32_t t_end = sat(tokens, group_sum((uint32_t)max(n, 0), tot));
    const uint32_t t_start = t_end - (uint32_t)max(n, 0);  // (not where the sum has stopped: refused below)
    const int64_t after = (int64_t)L + n;
    const int before_pages = L >= 0 ? pages_of(L) : 0;
    bool fine = mine && L >= 0 && n >= 0 && pages_of(after) <= p.max_pages && t_end <= (uint32_t)p.max_tokens && t_end < kMost;
    const uint32_t need = fine ? (uint32_t)(pages_of(after) - before_pages) : 0;
    const uint32_t p_end = sat(pages, group_sum(need, tot));
    fine = fine && (need == 0 || p_end <= free);
    const uint32_t granted = fine ? need : 0;
    if constexpr (WHAT & 2) {
      if (first_group && mine) p.seq_lens_out[b] = fine ? (int)after : L;
    }
    if constexpr (WHAT & 1) {
      if (first_group && mine) {
        p.q_start[b + 1] = (int)t_end;
        if (b == 0) p.q_start[0] = 0;
      }
    }
    token_end[tid] = t_end;
    page_end[tid] = p_end;
    had[tid] = fine ? before_pages : -1;
    len[tid] = L;
    // (whether all of the chunk's requests bring one token at most: a decode step)
    const bool chunky = __syncthreads_or(n > 1);
    const int last = min(threads, p.batch - b0) - 1;
    if constexpr (WHAT & 1) {
      if (!chunky) {
        if (first_group && mine && n == 1 && t_end <= (uint32_t)p.max_tokens) {
          int slot = -1;
          if (fine) {
            const int page = granted ? p.free_pages[free - p_end] : start_page;
            if (granted) p.page_table[b * p.stride + before_pages] = page;
            slot = page * kPage + L % kPage;
          }
          p.slot_map[t_start] = slot;
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
    __syncthreads();  // the sums are read before the next chunk's replace them
  }
  if constexpr (WHAT & 1) {
    for (uint32_t i = tokens + blockIdx.x * threads + tid; i < (uint32_t)p.max_tokens; i += gridDim.x * threads) p.slot_map[i] = -1;
  }
  if constexpr (WHAT & 2) {
    if (first_group) {
      for (int d = 1; d < 64; d *= 2) used = max(used, (uint32_t)__shfl_xor(used, d));
      if ((tid & 63) == 0) tot[tid >> 6] = used;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < threads / 64; ++w) used = max(used, tot[w]);
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
    const uint32_t end = sat(pages, group_sum((uint32_t)min(pages_of(max(L, 0)), p.max_pages), tot));
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
  // Work groups: one for each 1024 slots.
  const int want = std::max(p.batch, std::min(p.max_tokens, kThreads));
  const int threads = std::min(kThreads, (want + 63) / 64 * 64);
  const int groups = std::max(1, std::min(256, (p.max_tokens + threads - 1) / threads));
  const bool in_place = p.seq_lens_out == p.seq_lens || p.free_count_out == p.free_count;
  if (in_place && groups > 1) {
    hipLaunchKernelGGL(extend_kernel<1>, dim3(groups), dim3(threads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(extend_kernel<2>, dim3(1), dim3(threads), 0, stream, p);
  } else {
    hipLaunchKernelGGL(extend_kernel<3>, dim3(groups), dim3(threads), 0, stream, p);
  }
  return hipGetLastError();
}

hipError_t launch_table_release(const ReleaseParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace omniattn
