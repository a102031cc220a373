// Which drafted tokens stay.
//
// Node i of a request's tree has the target's logits l for the token behind it; p = softmax(l / T).  A token y is chosen for every node by
// itself, so that all rows of the call are looked at in parallel; the walk from node 0 to the child that holds y, and so on, comes last.
//   T = 0:           y = argmax l, the first of equals.
//   no draft's q:    y = the first v with p_0 + .. + p_v > u1 (p_0 + .. + p_V-1).
//   q given:         the node's first child x was drawn from q.  It is taken if u0 q(x) < p(x); otherwise y is found as above with max(p - q, 0)
//                    in p's place, so that y is distributed as p either way (where that is 0 everywhere, p itself).
// A child that holds y (the first such) is next; without one, y is the text's new last token.
//
// Sums and exponentials are in 64 bits: a border between two tokens that is off by 2^-24 of the whole gives another token once in some
// thousand draws from a large vocabulary, and then the same inputs would give other tokens with another order of summation.
//
// Kernels: sums of 2048 columns each; with q, what becomes of first children, and the sums of max(p - q, 0) of rows that need them; the
// nodes' tokens (a wave finds the part of 2048 columns whose running sum passes the border, and looks at these again); the walk.  Logits are read
// once, but for the parts that tokens are found in and, with q, the rows whose first child is refused.
//
// What bounds them: the sums, in bf16, the exponentials (13 instructions of 64 bits for a logit, about 5 clocks each; 64 requests of 6
// nodes, 131072 columns: 38 us, 2.6 TB/s, 20.3 vector instructions of all kinds a logit; vector units at work 84 % of the time); in fp32 memory nearly
// (32 requests of 40 nodes, 100003 columns: 97 us, 5.3 TB/s; maxima alone 89; vector units 87 %).  The kernels behind them take 5 to 14 us each, which are chains of loads; a node's part costs 2 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "verify.h"
#include "wave.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;  // (rows begin where they will)

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPickThreads = 512;
constexpr int kNodes = OMNIATTN_TREE_NODES;
// A wave looks at tiles of its columns, 16 bytes of neighbouring logits to a lane.
template <typename T>
struct Tile {
  static constexpr int kEach = 16 / sizeof(T), kColumns = 64 * kEach, kMany = kVerifyColumns / kColumns;
};
constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;
constexpr double kLeast = -1020.0;

// How a request's logits become weights 2^(c (l - top)): c, and the distance from which on they are taken for this distance (a weight of 2^kLeast, which no
// sum of a row notices).
struct Scale {
  double c, least;
};
// (A request without a temperature takes the likeliest token; its probabilities are those at 1.  An infinite one: c is not 0, or -inf would get a weight.)
__device__ __forceinline__ Scale scale_of(float T) {
  const double c = T > 0.f ? fmax(kLog2e / (double)T, 0x1p-1000) : kLog2e, inverse = T > 0.f ? fmin(kLn2 * (double)T, 0x1p+1000) : kLn2;
  return Scale{c, kLeast * inverse};
}
// 2^(c d) for d <= 0 (NaN: as for `least`), by rounding c d to an integer: by adding and taking away 1.5 * 2^52, in whose low word the integer then stands.
// (The instructions for that, for the conversion and for the scaling take longer than an addition, which takes twice as long as in 32 bits.)
constexpr double kMagic = 6755399441055744.0;
// 2^f 2^n for f in [-1/2, 1/2] and n in the low word of t.  Of the polynomials of degree 7 that are 1 at 0 the one that is off by the least part of 2^f: by
// 4.7e-11.  (1 at 0, so that the largest logits' weights are 1: sums of tokens that are equally likely are exact then, and a u1 on the border between
// two of them gives the one behind it.)
__device__ __forceinline__ double power_of(double f, double t) {
  double y = 1.519615685518997e-05;
  y = fma(y, f, 1.5466756311730684e-04);
  y = fma(y, f, 1.333393505442565e-03);
  y = fma(y, f, 9.6180381320883e-03);
  y = fma(y, f, 5.550410365992507e-02);
  y = fma(y, f, 2.402265106656079e-01);
  y = fma(y, f, 6.931471807045319e-01);
  y = fma(y, f, 1.0);
  // (asked for by name: the compiler makes a sum of 64 bits of it, in five instructions)
  u32x2 bits = __builtin_bit_cast(u32x2, y);
  asm("v_lshl_add_u32 %0, %1, 20, %0" : "+v"(bits[1]) : "v"(__builtin_bit_cast(u32x2, t)[0]));
  return __builtin_bit_cast(double, bits);
}
__device__ __forceinline__ double power(double d, const Scale& s) {
  d = fmax(d, s.least);
  const double t = fma(d, s.c, kMagic);
  return power_of(fma(d, s.c, kMagic - t), t);
}
// Weight of a logit beside the largest.
__device__ __forceinline__ double weight(float l, double top, const Scale& s) { return power((double)l - top, s); }
// The same, 0 where there is none.
__device__ __forceinline__ double weight_or_0(float l, double top, const Scale& s) {
  const double d = (double)l - top;
  return d > s.least ? power(d, s) : 0.0;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ double readlane64(double x, int lane) {
  const int64_t v = __builtin_bit_cast(int64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane);
  return __builtin_bit_cast(double, (int64_t)((uint64_t)hi << 32 | lo));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved64(double x) {  // (0 where nothing comes from)
  const int64_t v = __builtin_bit_cast(int64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, true);
  return __builtin_bit_cast(double, (int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double wave_sum_up_to(double x) {
  x += moved64<0x111, 0xf>(x);  // from the lane one, two, four, eight before, in rows of 16
  x += moved64<0x112, 0xf>(x);
  x += moved64<0x114, 0xf>(x);
  x += moved64<0x118, 0xf>(x);
  x += moved64<0x142, 0xa>(x);  // a row's last lane to the row behind it
  x += moved64<0x143, 0xc>(x);  // lane 31 to the upper half
  return x;
}
__device__ __forceinline__ double wave_sum(double x) { return readlane64(wave_sum_up_to(x), 63); }
__device__ __forceinline__ float wave_max(float x) {
  return __builtin_bit_cast(float, wave_join(__builtin_bit_cast(uint32_t, x), [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  }));
}
__device__ __forceinline__ int wave_min(int x) {
  return (int)wave_join((uint32_t)x, [](uint32_t a, uint32_t b) { return (uint32_t)min((int)a, (int)b); });
}

struct Nodes {
  int begin, n;
};
__device__ __forceinline__ Nodes nodes_of(const VerifyParams& p, int b) {
  const int lo = p.q_start ? p.q_start[b] : b, hi = p.q_start ? p.q_start[b + 1] : b + 1;
  Nodes r;
  r.begin = min(max(lo, 0), p.num_tokens);
  r.n = min(max(hi, r.begin), p.num_tokens) - r.begin;
  return r;
}
// The request that row `row` of the call belongs to, or -1, and its temperature.
struct Owner {
  int b;
  float T;
};
__device__ __forceinline__ Owner owner_of(const VerifyParams& p, int row) {
  if (!p.q_start) return row < p.batch ? Owner{row, p.temperature[row]} : Owner{-1, 0.f};
  const int lane = threadIdx.x & 63, first = p.q_start[0];
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const int b = min(b0 + lane, p.batch - 1);
    const float T = p.temperature[b];
    const uint64_t beyond = __ballot(p.q_start[b + 1] > row);
    if (!beyond) continue;
    const int i = __builtin_ctzll(beyond);
    return row >= first ? Owner{b0 + i, __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, T), i))} : Owner{-1, 0.f};
  }
  return Owner{-1, 0.f};
}
// Neighbouring numbers of a row; those from column `stop` on are -inf.
template <typename T, int N>
__device__ __forceinline__ void load(float (&x)[N], const T* row, int col, int stop) {
  const T* at = row + col;
  if (col + N <= stop) {
#pragma unroll
    for (int k = 0; k < N; k += Tile<T>::kEach) {
      const u32x4 w = *(const u32x4_any*)(at + k);
#pragma unroll
      for (int i = 0; i < Tile<T>::kEach; ++i) {
        const uint32_t word = w[i * sizeof(T) / 4];
        if constexpr (sizeof(T) == 2) x[k + i] = __builtin_bit_cast(float, i % 2 ? word & 0xffff0000u : word << 16);
        else x[k + i] = __builtin_bit_cast(float, word);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2) x[i] = col + i < stop ? __builtin_bit_cast(float, (uint32_t)at[i] << 16) : -INFINITY;
      else x[i] = col + i < stop ? at[i] : -INFINITY;
    }
  }
}
template <typename T>
__device__ __forceinline__ const T* logits_of(const VerifyParams& p, int row) { return (const T*)p.logits + row * p.stride; }

// Maxima without the instructions by which the compiler makes sure that a signalling NaN counts as no number: with one the result is NaN.
__device__ __forceinline__ float max2(float x, float y) {
  float z;
  asm("v_max_f32 %0, %1, %2" : "=v"(z) : "v"(x), "v"(y));
  return z;
}
__device__ __forceinline__ float max3(float x, float y, float z) {
  asm("v_max3_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z));
  return x;
}

// A wave's kVerifyColumns columns of a row, as they lie in memory; behind the row's end -inf.
template <typename T>
struct Columns {
  using Of = Tile<T>;
  u32x4 w[Of::kMany];
  __device__ __forceinline__ float at(int t, int i) const {
    const uint32_t word = w[t][i * sizeof(T) / 4];
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, i % 2 ? word & 0xffff0000u : word << 16);
    else return __builtin_bit_cast(float, word);
  }
  __device__ __forceinline__ void fetch(const T* row, int part, int vocab) {
    const int col = part * kVerifyColumns + (threadIdx.x & 63) * Of::kEach;
    if ((part + 1) * kVerifyColumns <= vocab) {
#pragma unroll
      for (int t = 0; t < Of::kMany; ++t) w[t] = *(const u32x4_any*)(row + col + t * Of::kColumns);
    } else {
#pragma unroll
      for (int t = 0; t < Of::kMany; ++t) {
        float x[Of::kEach];
        load<T>(x, row, col + t * Of::kColumns, vocab);
#pragma unroll
        for (int i = 0; i < Of::kEach; ++i) {
          const uint32_t bits = __builtin_bit_cast(uint32_t, x[i]);
          if constexpr (sizeof(T) == 2) w[t][i / 2] = i % 2 ? w[t][i / 2] | bits : bits >> 16;
          else w[t][i] = bits;
        }
      }
    }
  }
};

// A wave to kVerifyColumns columns of a row.
template <typename T>
__global__ __launch_bounds__(kThreads, 8) void verify_sums_kernel(VerifyParams p) {
  using Of = Tile<T>;
  const int lane = threadIdx.x & 63;
  const uint32_t id = blockIdx.x * kWaves + uniform(threadIdx.x >> 6), row = id / (uint32_t)p.num_parts, part = id - row * p.num_parts;
  if (row >= (uint32_t)p.num_tokens) return;
  Columns<T> x;
  x.fetch(logits_of<T>(p, row), part, p.vocab);
  const Owner owner = owner_of(p, row);
  if (owner.b < 0) return;
  const Scale c = scale_of(owner.T);
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < Of::kMany; ++t)
#pragma unroll
    for (int i = 0; i < Of::kEach; i += 2) top = max3(top, x.at(t, i), x.at(t, i + 1));
  top = wave_max(top);
  double m = top, sum = 0.0;
  if (fabs(m * c.c) < 0x1p+30 && c.c > 1e-30) {
    // (with `least` in 32 bits: off by 2^-24 of a product below 2^31, by 128 at most)
    const float least = (float)fma(c.least, (kLeast + 160.0) / kLeast, m);
#pragma unroll
    for (int t = 0; t < Of::kMany; ++t)
#pragma unroll
      for (int i = 0; i < Of::kEach; ++i) {
        const double d = (double)max2(x.at(t, i), least) - m, n = fma(d, c.c, kMagic);
        sum += power_of(fma(d, c.c, kMagic - n), n);
      }
    asm volatile("" : "+v"(sum));  // (added up here: behind a condition the compiler keeps all the weights until there, in the room of half of the waves)
    sum = wave_sum(sum);
  } else {
    sum = NAN;
  }
  if (!(sum > 0.0)) {  // signalling NaN, infinities, extreme temperatures
    top = -INFINITY;
#pragma unroll
    for (int t = 0; t < Of::kMany; ++t)
#pragma unroll
      for (int i = 0; i < Of::kEach; ++i) top = fmaxf(top, x.at(t, i));
    top = wave_max(top);
    m = top;
    sum = 0.0;
#pragma unroll
    for (int t = 0; t < Of::kMany; ++t)
#pragma unroll
      for (int i = 0; i < Of::kEach; ++i) sum += weight(x.at(t, i), m, c);
    asm volatile("" : "+v"(sum));
    sum = fabsf(top) < INFINITY ? wave_sum(sum) : 0.0;
  }
  int best = 0x7fffffff;
  if (!(owner.T > 0.f) || top == INFINITY) {
#pragma unroll
    for (int t = Of::kMany - 1; t >= 0; --t)
#pragma unroll
      for (int i = Of::kEach - 1; i >= 0; --i)
        if (x.at(t, i) == top) best = part * kVerifyColumns + t * Of::kColumns + lane * Of::kEach + i;
    best = wave_min(best);
  }
  if (lane == 0) p.parts[(size_t)row * p.num_parts + part] = VerifyPart{sum, top, best};
}

// A row's parts, two neighbours to a lane: part k0 + 2 lane + i.
struct Pair {
  VerifyPart e[2];
};
__device__ __forceinline__ Pair pair_of(const VerifyParams& p, int row, int k0) {
  const VerifyPart* const parts = p.parts + (size_t)row * p.num_parts;
  Pair r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = k0 + 2 * (threadIdx.x & 63) + i;
    r.e[i] = parts[min(k, p.num_parts - 1)];
    if (k >= p.num_parts) r.e[i] = VerifyPart{0.0, -INFINITY, 0x7fffffff};
  }
  return r;
}
// A row's largest logit, the first column that has it, and the sum of its weights.
struct Row {
  double top, sum;
  float ftop;
  int best;
};
__device__ __forceinline__ Row row_of(const VerifyParams& p, int row, const Pair& first, const Scale& c) {
  Row r;
  float top = -INFINITY;
  double sum = 0.0;
  int best = 0x7fffffff;
  Pair at = first;
  for (int k0 = 0; k0 < p.num_parts; k0 += 128) {
    if (k0) at = pair_of(p, row, k0);
    const float next = fmaxf(top, fmaxf(at.e[0].top, at.e[1].top));
    sum *= weight(top, next, c);
    if (next > top) best = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum += at.e[i].sum * weight(at.e[i].top, next, c);
      if (at.e[i].top == next) best = min(best, at.e[i].best);
    }
    top = next;
  }
  r.ftop = wave_max(top);
  r.top = r.ftop;
  r.sum = wave_sum(sum * weight(top, r.top, c));
  r.best = wave_min(top == r.ftop ? best : 0x7fffffff);
  return r;
}
// Probability of a logit in a row, in whose column `col` it is.  (Rows with infinite logits: the first such token has all.)
__device__ __forceinline__ double chance_of(const Row& r, double inverse, float l, int col, const Scale& c) {
  if (r.ftop == INFINITY) return col == r.best ? 1.0 : 0.0;
  return weight_or_0(l, r.top, c) * inverse;
}
__device__ __forceinline__ double inverse_of(const Row& r) { return r.sum > 0.0 ? 1.0 / r.sum : 0.0; }

// With drafts' probabilities: a wave to a row.  Its sums, its first child, and whether that is taken.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_rows_kernel(VerifyParams p) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (row >= p.num_tokens) return;
  const Pair first = pair_of(p, row, 0);
  const Owner owner = owner_of(p, row);
  if (owner.b < 0) return;
  const Nodes r = nodes_of(p, owner.b);
  if (r.n > kNodes) return;
  const int node = row - r.begin, parent = lane < r.n ? p.parents[r.begin + lane] : -1, token = lane < r.n ? p.tokens[r.begin + lane] : -1;
  const Scale c = scale_of(owner.T);
  VerifyRow out;
  const Row all = row_of(p, row, first, c);
  out.sum = all.sum;
  out.top = all.ftop;
  out.best = all.best;
  const uint64_t children = owner.T > 0.f ? __ballot(lane > node && parent == node) : 0;
  out.child = children ? __builtin_ctzll(children) : -1;
  out.taken = 0;
  out.logit = -INFINITY;
  if (children) {
    const int x = __builtin_amdgcn_readlane(token, out.child);
    if ((uint32_t)x < (uint32_t)p.vocab) {
      const T* const at = logits_of<T>(p, row) + x;
      if constexpr (sizeof(T) == 2) out.logit = __builtin_bit_cast(float, (uint32_t)*at << 16);
      else out.logit = *at;
      out.taken = (double)p.uniforms[2 * (int64_t)row] * (double)p.draft_probs[row * p.draft_stride + x] < chance_of(all, inverse_of(all), out.logit, x, c);
    }
  }
  if (lane == 0) p.rows[row] = out;
}
// Nodes that the walk is likely to come to: it goes to a first child that is taken, and to others if it is not.  (To a first child that is not taken
// only if nothing is left of max(p - q, 0): the walk has such nodes looked at when it comes to them.)  Lane a has node a.
__device__ __forceinline__ bool reached(int node, int parent, const VerifyRow& mine) {
  const int lane = threadIdx.x & 63, of = parent >= 0 && parent < lane ? parent : 0;
  const bool first = __shfl(mine.child, of) == lane, taken = __shfl(mine.taken, of) != 0;
  const uint64_t open = __ballot(parent >= 0 && parent < lane && first == taken);
  while (node > 0) {
    if (!(open >> node & 1)) return false;
    node = __builtin_amdgcn_readlane(parent, node);
  }
  return true;
}
// max(p - q, 0) of neighbours, and their logits.
template <typename T, int N>
__device__ __forceinline__ void rest_of(double (&w)[N], float (&x)[N], const VerifyParams& p, const Row& r, double inverse, int row, int col, const Scale& c) {
  float q[N];
  load<T>(x, logits_of<T>(p, row), col, p.vocab);
  load<float>(q, p.draft_probs + row * p.draft_stride, col, p.vocab);
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = col + i < p.vocab ? fmax(chance_of(r, inverse, x[i], col + i, c) - (double)q[i], 0.0) : 0.0;
}
__device__ __forceinline__ Row row_of(const VerifyRow& r) { return Row{(double)r.top, r.sum, r.top, r.best}; }
__device__ __forceinline__ float readlane_f(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }
// What lane `lane` holds.
__device__ __forceinline__ VerifyRow row_at(const VerifyRow& r, int lane) {
  return VerifyRow{readlane64(r.sum, lane), readlane_f(r.top, lane), __builtin_amdgcn_readlane(r.best, lane), __builtin_amdgcn_readlane(r.child, lane),
                   __builtin_amdgcn_readlane(r.taken, lane), readlane_f(r.logit, lane)};
}

// Of kVerifyColumns columns of a row.
template <typename T>
__device__ __forceinline__ void rest_of_part(const VerifyParams& p, const Row& r, double inverse, int row, int part, const Scale& c) {
  const int lane = threadIdx.x & 63;
  double sum = 0.0;
#pragma unroll
  for (int t = 0; t < Tile<T>::kMany; ++t) {
    double w[Tile<T>::kEach];
    float x[Tile<T>::kEach];
    rest_of<T>(w, x, p, r, inverse, row, part * kVerifyColumns + t * Tile<T>::kColumns + lane * Tile<T>::kEach, c);
#pragma unroll
    for (int i = 0; i < Tile<T>::kEach; ++i) sum += w[i];
  }
  sum = wave_sum(sum);
  if (lane == 0) p.rest[(size_t)row * p.num_parts + part] = sum;
}

// Sums of max(p - q, 0), of the rows whose first child is not taken and that the walk is likely to come to (of a chain: one).  `slices` work groups to a request,
// a wave to every so many parts of kVerifyColumns columns.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_rest_kernel(VerifyParams p, int slices) {
  const int lane = threadIdx.x & 63, b = blockIdx.x / slices, wave = (blockIdx.x - b * slices) * kWaves + uniform(threadIdx.x >> 6);
  const float T0 = p.temperature[b];
  const Nodes r = nodes_of(p, b);
  if (!(T0 > 0.f) || r.n > kNodes || r.n == 0) return;
  const int at = r.begin + min(lane, r.n - 1), parent = p.parents[at];
  const VerifyRow mine = p.rows[at];
  const Scale c = scale_of(T0);
  for (uint64_t refused = __ballot(lane < r.n && mine.child >= 0 && !mine.taken); refused; refused &= refused - 1) {
    const int node = __builtin_ctzll(refused), row = r.begin + node;
    if (!reached(node, parent, mine)) continue;
    const Row all = row_of(row_at(mine, node));
    const double inverse = inverse_of(all);
    for (int part = wave; part < p.num_parts; part += slices * kWaves) rest_of_part<T>(p, all, inverse, row, part, c);
  }
}

struct Found {
  int col;      // -1: no column has a weight
  float logit;
};
// First column at which the running sum of a row's weights is above `border`.  part_sums(k0): of parts k0 + 2 lane + i; weights(w, x, col): of a lane's
// neighbours in a tile.  (The last column with a weight if rounding leaves none above the border.)
template <typename T, typename F, typename G>
__device__ __forceinline__ Found find(const VerifyParams& p, double border, F part_sums, G weights) {
  constexpr int kMany = Tile<T>::kMany, kEach = Tile<T>::kEach;
  const int lane = threadIdx.x & 63;
  double before = 0.0, run = 0.0;
  int part = -1;
  for (int k0 = 0; k0 < p.num_parts; k0 += 128) {
    const double2 s = part_sums(k0);
    const double upto = wave_sum_up_to(s.x + s.y), here = before + upto - (s.x + s.y), middle = here + s.x;
    const uint64_t hit0 = __ballot(s.x > 0.0 && middle > border), hit1 = __ballot(s.y > 0.0 && before + upto > border);
    const uint64_t some0 = __ballot(s.x > 0.0), some1 = __ballot(s.y > 0.0);
    if (hit0 | hit1) {
      const int i = __builtin_ctzll(hit0 | hit1);
      const bool second = !(hit0 >> i & 1);
      part = k0 + 2 * i + second;
      run = readlane64(second ? middle : here, i);
      break;
    }
    if (some0 | some1) {
      const int i = 63 - __builtin_clzll(some0 | some1);
      const bool second = some1 >> i & 1;
      part = k0 + 2 * i + second;
      run = readlane64(second ? middle : here, i);
    }
    before += readlane64(upto, 63);
  }
  if (part < 0) return Found{-1, 0.f};
  double w[kMany][kEach], upto[kMany], s[kMany];
  float x[kMany][kEach];
  const int col = part * kVerifyColumns + lane * kEach;
#pragma unroll
  for (int t = 0; t < kMany; ++t) {
    weights(w[t], x[t], col + t * Tile<T>::kColumns);
    s[t] = (w[t][0] + w[t][1]) + (w[t][2] + w[t][3]);
    if constexpr (kEach == 8) s[t] += (w[t][4] + w[t][5]) + (w[t][6] + w[t][7]);
  }
#pragma unroll
  for (int t = 0; t < kMany; ++t) upto[t] = wave_sum_up_to(s[t]);
  Found last = {-1, 0.f};
#pragma unroll
  for (int t = 0; t < kMany; ++t) {
    double sum = run + upto[t] - s[t];
    int hit = -1, mine = -1;
    float hit_logit = 0.f, my_logit = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      sum += w[t][i];
      if (w[t][i] > 0.0) {
        mine = col + t * Tile<T>::kColumns + i;
        my_logit = x[t][i];
        if (sum > border && hit < 0) {
          hit = mine;
          hit_logit = my_logit;
        }
      }
    }
    const uint64_t hits = __ballot(hit >= 0), some = __ballot(mine >= 0);
    if (hits) {
      const int i = __builtin_ctzll(hits);
      return Found{__builtin_amdgcn_readlane(hit, i), __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, hit_logit), i))};
    }
    if (some) {
      const int i = 63 - __builtin_clzll(some);
      last = Found{__builtin_amdgcn_readlane(mine, i), __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_logit), i))};
    }
    run += readlane64(upto[t], 63);
  }
  return last;
}

// The token of node `node` of a request, the child that the walk goes to (-1: none; kUnseen: not looked at), and the logarithm of the token's
// probability.  A wave; lane a knows parent and token of node a.  asked: the walk has come to it.
constexpr int kUnseen = -2;
template <typename T, bool DRAFTS>
__device__ __forceinline__ VerifyChoice choose(const VerifyParams& p, const Nodes& r, int node, float T0, int parent, int token, bool asked) {
  const int lane = threadIdx.x & 63, row = r.begin + node;
  const Scale c = scale_of(T0);
  const uint64_t children = __ballot(lane > node && lane < r.n && parent == node);
  const Pair first = pair_of(p, row, 0);
  const float u = p.uniforms[2 * (int64_t)row + 1];
  const bool drafted = DRAFTS && T0 > 0.f && children;
  Row all;
  VerifyRow kept;
  if constexpr (DRAFTS) {
    const VerifyRow mine = p.rows[r.begin + min(lane, r.n - 1)];
    if (!reached(node, parent, mine)) {
      if (!asked) return VerifyChoice{-1, kUnseen, 0.f};
    } else {
      asked = false;
    }
    kept = row_at(mine, node);
    all = row_of(kept);
  } else {
    all = row_of(p, row, first, c);
  }
  VerifyChoice out = {-1, -1, 0.f};
  Found y = {-1, 0.f};
  if (!(T0 > 0.f) || all.ftop == INFINITY) y = Found{all.ftop == -INFINITY ? -1 : all.best, all.ftop};
  if (drafted && kept.taken) {
    out.next = kept.child;
    y = Found{__builtin_amdgcn_readlane(token, kept.child), kept.logit};
  } else if (T0 > 0.f) {
    bool found = false;
    if (drafted) {
      if (asked) {
        for (int part = 0; part < p.num_parts; ++part) rest_of_part<T>(p, all, inverse_of(all), row, part, c);
        __threadfence();
      }
      const double* const rest = p.rest + (size_t)row * p.num_parts;
      auto part_sums = [&](int k0) {
        const int k = k0 + 2 * lane;
        return double2{k < p.num_parts ? rest[k] : 0.0, k + 1 < p.num_parts ? rest[k + 1] : 0.0};
      };
      double sum = 0.0;
      for (int k0 = 0; k0 < p.num_parts; k0 += 128) {
        const double2 s = part_sums(k0);
        sum += s.x + s.y;
      }
      sum = wave_sum(sum);
      if (sum > 0.0) {
        const double inverse = inverse_of(all);
        y = find<T>(p, (double)u * sum, part_sums, [&](auto& w, auto& x, int col) { rest_of<T>(w, x, p, all, inverse, row, col, c); });
        found = true;
      }
    }
    if (!found && all.ftop < INFINITY && all.sum > 0.0) {
      y = find<T>(p, (double)u * all.sum,
               [&](int k0) {
                 const Pair at = k0 ? pair_of(p, row, k0) : first;
                 // (nothing where the part's largest logit has no weight: find is to come to parts with a column that has one)
                 return double2{at.e[0].sum * weight_or_0(at.e[0].top, all.top, c), at.e[1].sum * weight_or_0(at.e[1].top, all.top, c)};
               },
               [&](auto& w, auto& x, int col) {
                 load<T>(x, logits_of<T>(p, row), col, p.vocab);
#pragma unroll
                 for (int i = 0; i < Tile<T>::kEach; ++i) w[i] = weight_or_0(x[i], all.top, c);
               });
    }
  }
  out.token = y.col;
  if (y.col < 0) return out;
  if (out.next < 0) {
    const uint64_t same = children & __ballot(token == y.col);
    if (same) out.next = __builtin_ctzll(same);
  }
  if (all.ftop == INFINITY) out.logprob = y.col == all.best ? 0.f : -INFINITY;
  else out.logprob = (float)((((double)y.logit - all.top) * c.c - log2(all.sum)) * kLn2);
  return out;
}

// Down the tree.  A wave; lane a knows node a's choice.
struct Way {
  int kept, node;  // how many nodes, and lane i's: the i-th of them (-1: none)
  int unseen;      // a node on it that was not looked at, or -1
};
__device__ __forceinline__ Way way_of(const Nodes& r, const VerifyChoice& mine) {
  const int lane = threadIdx.x & 63;
  Way w = {0, -1, -1};
  for (int at = r.n > 0 ? 0 : -1; at >= 0;) {  // (a child's number is above its parent's)
    const int next = __builtin_amdgcn_readlane(mine.next, at);
    if (lane == w.kept) w.node = at;
    ++w.kept;
    if (next == kUnseen) w.unseen = at;
    at = next;
  }
  return w;
}
// The request's results.
__device__ __forceinline__ void write(const VerifyParams& p, int b, const Nodes& r, const Way& way, const VerifyChoice& mine) {
  const int lane = threadIdx.x & 63, node = way.node;
  const int token = __shfl(mine.token, max(node, 0));
  const float logprob = __shfl(mine.logprob, max(node, 0));
  if (lane < r.n) {
    p.path[r.begin + lane] = node;
    p.out_tokens[r.begin + lane] = node >= 0 ? token : -1;
    if (p.logprobs) p.logprobs[r.begin + lane] = node >= 0 ? logprob : 0.f;
  }
  if (lane == 0) p.dropped[b] = r.n - way.kept;
}
// A request with too many nodes keeps none.
__device__ __forceinline__ void keep_none(const VerifyParams& p, int b, const Nodes& r) {
  for (int t = threadIdx.x; t < r.n; t += blockDim.x) {
    p.path[r.begin + t] = -1;
    p.out_tokens[r.begin + t] = -1;
    if (p.logprobs) p.logprobs[r.begin + t] = 0.f;
  }
  if (threadIdx.x == 0) p.dropped[b] = r.n;
}

// Trees of few nodes, or with drafts' probabilities: a work group to a request, whose waves choose the nodes' tokens; then one walks down the tree.
template <typename T, bool DRAFTS>
__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(VerifyParams p) {
  __shared__ VerifyChoice choices[kNodes];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), b = blockIdx.x;
  const Nodes r = nodes_of(p, b);
  if (r.n > kNodes) return keep_none(p, b, r);
  const float T0 = p.temperature[b];
  const int parent = lane < r.n ? p.parents[r.begin + lane] : -1, token = lane < r.n ? p.tokens[r.begin + lane] : -1;
  for (int first = wave, end = r.n, asked = false;; asked = true) {
    for (int i = first; i < end; i += kPickThreads / 64) {
      const VerifyChoice choice = choose<T, DRAFTS>(p, r, i, T0, parent, token, asked);
      if (lane == 0) choices[i] = choice;
    }
    __syncthreads();
    const VerifyChoice mine = choices[min(lane, max(r.n - 1, 0))];
    const Way way = way_of(r, mine);
    if (!DRAFTS || way.unseen < 0) {
      if (wave == 0) write(p, b, r, way, mine);
      break;
    }
    first = way.unseen + wave;  // (by the first wave)
    end = way.unseen + 1;
    __syncthreads();
  }
}
// Trees of many: a wave to a node of the call; and then a wave to a request.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_choose_kernel(VerifyParams p) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  if (row >= p.num_tokens) return;
  const Owner owner = owner_of(p, row);
  if (owner.b < 0) return;
  const Nodes r = nodes_of(p, owner.b);
  if (r.n > kNodes) return;
  const int parent = lane < r.n ? p.parents[r.begin + lane] : -1, token = lane < r.n ? p.tokens[r.begin + lane] : -1;
  const VerifyChoice choice = choose<T, false>(p, r, row - r.begin, owner.T, parent, token, false);
  if (lane == 0) p.choices[row] = choice;
}
__global__ __launch_bounds__(64) void verify_walk_kernel(VerifyParams p) {
  const int b = blockIdx.x, lane = threadIdx.x;
  const Nodes r = nodes_of(p, b);
  if (r.n > kNodes) return keep_none(p, b, r);
  const VerifyChoice mine = lane < r.n ? p.choices[r.begin + lane] : VerifyChoice{-1, -1, 0.f};
  write(p, b, r, way_of(r, mine), mine);
}

template <typename T, bool DRAFTS>
hipError_t start(const VerifyParams& p, int cus, hipStream_t stream) {
  if (p.num_tokens > 0) {
    const dim3 by_row((p.num_tokens + kWaves - 1) / kWaves);
    const int64_t groups = ((int64_t)p.num_tokens * p.num_parts + kWaves - 1) / kWaves;
    hipLaunchKernelGGL(verify_sums_kernel<T>, dim3((uint32_t)groups), dim3(kThreads), 0, stream, p);
    if constexpr (DRAFTS) {
      const int slices = std::max(1, std::min((p.num_parts + kWaves - 1) / kWaves, 8 * cus / p.batch));
      hipLaunchKernelGGL(verify_rows_kernel<T>, by_row, dim3(kThreads), 0, stream, p);
      hipLaunchKernelGGL(verify_rest_kernel<T>, dim3((uint32_t)p.batch * slices), dim3(kThreads), 0, stream, p, slices);
    }
    // More nodes to a request (their mean, which the host knows) than a work group has waves take turns there, which costs more than a second launch.
    // With drafts' probabilities few of them are looked at, and a work group to a request is as fast for trees of any size.  us a call, bf16, work
    // group to a request / wave to a node (vocabulary x requests; "q": drafts' probabilities given):
    //   nodes             6             8             9            16            32            64
    //    32000 x 1    12.4 / 13.6   12.9 / 13.8   16.3 / 13.9   19.7 / 13.8   32.6 / 14.1   57.5 / 14.3
    //    32000 x 64   20.3 / 21.3   24.6 / 25.8   30.3 / 28.2   43.1 / 38.0   76.0 / 58.3    137 / 106
    //   131072 x 64   44.1 / 45.9   52.4 / 53.9   61.0 / 58.1   94.1 / 90.6    193 / 185     371 / 355
    //   q 32000 x 1   23.2 / 25.0   23.3 / 25.0   23.3 / 25.1   24.5 / 25.7   26.4 / 26.5   31.4 / 28.7
    //   q 32000 x 64  34.7 / 37.8   38.6 / 41.9   40.9 / 44.2   51.7 / 53.4   72.2 / 73.2    113 / 117
    //   q131072 x 64  63.4 / 66.9   73.0 / 75.5   76.4 / 79.5    114 / 117     199 / 199     369 / 370
    if constexpr (!DRAFTS) {
      if (p.num_tokens > (int64_t)p.batch * (kPickThreads / 64)) {
        hipLaunchKernelGGL(verify_choose_kernel<T>, by_row, dim3(kThreads), 0, stream, p);
        hipLaunchKernelGGL(verify_walk_kernel, dim3(p.batch), dim3(64), 0, stream, p);
        return hipGetLastError();
      }
    }
  }
  hipLaunchKernelGGL((verify_pick_kernel<T, DRAFTS>), dim3(p.batch), dim3(kPickThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_verify(const VerifyParams& p, int cus, hipStream_t stream) {
  if (p.draft_probs) return p.logits_fp32 ? start<float, true>(p, cus, stream) : start<uint16_t, true>(p, cus, stream);
  return p.logits_fp32 ? start<float, false>(p, cus, stream) : start<uint16_t, false>(p, cus, stream);
}

}  // namespace omniattn
