// How the attention kernels of the grouped-query part deal out their work, as far as it needs no GPU: the blocks of query rows and what they
// cost, the shares, and the walk from block to block.  (Plain C++, so that it can be run on the host for sizes that no GPU test reaches.)
// P: what the formulas need of a call, under the names of GqaDecodeParams.
#pragma once
#include <stdint.h>

#include "plan.h"

#if defined(__HIPCC__)
#define OA_INLINE __host__ __device__ __forceinline__
#else
#define OA_INLINE inline
#endif

namespace omniattn {

template <typename T>
OA_INLINE T lesser(T a, T b) { return a < b ? a : b; }
template <typename T>
OA_INLINE T larger(T a, T b) { return a > b ? a : b; }

// What a request brings: its tokens, its first query token and how many it has.
struct Request {
  int L, begin, n;
};
// Pages of a block of query rows (GRAIN 32: their quarters): the union of its queries' kept sets.
struct Block {
  int t0, t1;  // its query tokens, both included
  TileLayout pages;
};
// A block of up to 128 rows: how often a page is halved into units, so that a unit is the same steps of 32 rows and tokens whatever the rows (32 rows: 128
// tokens; 64: 64; more: 32).  (Not the same bytes: one of 32 rows has the codes of four of 128.)
template <int ROWS, typename P>
OA_INLINE int tree_split(const P& p, const Request& r, int rb) {
  if (ROWS < 128) return 0;
  const int rows = lesser(r.n * p.group - rb * ROWS, ROWS);
  return rows <= 32 ? 0 : rows <= 64 ? 1 : 2;
}

// TREE: the queries are nodes of a tree, of which any may see any, and which stand up to n - 1 tokens behind their positions: every block has the
// nodes' pages and all that a query at the first node's position keeps of the text.
template <int ROWS, int GRAIN, bool TREE = false, typename P>
OA_INLINE Block block_of(const P& p, const Request& r, int rb) {
  Block k;
  if constexpr (TREE) {
    k.t0 = 0;
    k.t1 = r.n - 1;
    const int text = r.L - r.n, grain = GRAIN >> tree_split<ROWS>(p, r, rb);
    // (without a window: the nodes that are sink tokens)
    k.pages = tile_layout(r.L, p.W == 0 && text < p.S ? p.S + OMNIATTN_TREE_NODES : p.S, p.W > 0 ? (int)lesser((int64_t)p.W + k.t1, (int64_t)larger(r.L, 1)) : 0, grain);
    return k;
  }
  // (rows of a call are counted in 32 bits; most requests have one block, and divisions are what a share's finding consists of)
  k.t0 = rb ? (int)((uint32_t)(rb * ROWS) / (uint32_t)p.group) : 0;
  k.t1 = (rb + 1) * ROWS >= r.n * p.group ? r.n - 1 : (int)((uint32_t)((rb + 1) * ROWS - 1) / (uint32_t)p.group);
  k.pages = tile_layout(r.L - r.n + k.t1 + 1, p.S, p.W > 0 ? p.W + (k.t1 - k.t0) : 0, GRAIN);
  return k;
}
template <int ROWS, typename P>
OA_INLINE int blocks_of(const P& p, const Request& r) {
  return (r.n * p.group + ROWS - 1) / ROWS;
}

// Share u of U: units [bound(u), bound(u + 1)), about u T / U.  Every share has T / U or one more; those with more are spread evenly (the
// neighbours in a compute unit would have a fifth more to read than others: 256 requests of 12 heads 33 us, in one run 40).
struct Shares {
  int64_t T, each;  // each = T / U
  int U;            // at most 2^14
  uint32_t more;    // (T % U) 2^17 / U, rounded up
  OA_INLINE Shares(int64_t total, int most) : T(total), U((int)lesser((int64_t)most, total)) {
    each = T >> 31 ? T / larger(U, 1) : (uint32_t)T / (uint32_t)larger(U, 1);
    more = ((uint32_t)(T - each * U) << 17) / (uint32_t)larger(U, 1) + 1;
  }
  OA_INLINE Shares() {}
  OA_INLINE int64_t bound(int u) const { return u * each + ((uint32_t)u * more >> 17); }
  // the share that has unit x
  OA_INLINE int owner(int64_t x) const {
    int u = lesser((int)((float)x * U / (float)T), U - 1);
    while (bound(u) > x) --u;
    while (bound(u + 1) <= x) ++u;
    return u;
  }
};

// The part of a block that belongs to a share.
struct Piece {
  int b, h, rb;
  Request rq;
  Block bk;
  int off;               // the block's units before it
  int tile_lo, tile_hi;  // its pages, by their number among the block's
  int64_t left;          // units of the share from its first one on
  OA_INLINE bool whole() const { return tile_lo == 0 && tile_hi == bk.pages.count(); }
  // tokens that query t sees: none if it comes before the request's first token (not a negative number, from which a window of nearly 2^31 tokens
  // could not be subtracted)
  OA_INLINE int reach(int t) const { return larger(rq.L - rq.n + t + 1, 0); }
};

// Walks through the blocks of a share.  R: rows of a block.  START: what a block costs beside its pages (its query, the meeting of the waves,
// its results), in pages or what GRAIN makes of them.
template <int R, int START, int GRAIN, typename P, bool TREE = false>
struct Walk {
  const P& p;
  OA_INLINE explicit Walk(const P& params) : p(params) {}

  OA_INLINE static int units(const Block& k) { return START + k.pages.count(); }
  OA_INLINE Block block(const Request& r, int rb) const { return block_of<R, GRAIN, TREE>(p, r, rb); }
  // Units of one KV head of a request
  OA_INLINE int64_t cost_of(const Request& r) const {
    const int blocks = blocks_of<R>(p, r);
    int64_t sum = 0;
    for (int rb = 0; rb < blocks; ++rb) sum += units(block(r, rb));
    return sum;
  }
  OA_INLINE void cut(Piece& w) const {
    w.bk = block(w.rq, w.rb);
    w.tile_lo = larger(w.off - START, 0);
    w.tile_hi = p.uncut ? w.bk.pages.count() : (int)lesser(larger(w.left + w.off - START, (int64_t)0), (int64_t)w.bk.pages.count());
  }
  // Whether there is something to do: pages, or the empty result of a block that keeps nothing, which is whose share has its first unit.
  OA_INLINE static bool counts(const Piece& w) { return w.tile_lo < w.tile_hi || (w.bk.pages.count() == 0 && w.off == 0); }
  // The next block of the share with something to do; false if there is none.  request(b): what request b brings.
  template <typename F>
  OA_INLINE bool follow(Piece& w, F request) const {
    do {
      w.left -= units(w.bk) - w.off;
      w.off = 0;
      if (w.left <= 0) return false;
      if (++w.rb >= blocks_of<R>(p, w.rq)) {
        w.rb = 0;
        if (++w.h == p.kv_heads) {
          w.h = 0;
          do w.rq = request(++w.b);
          while (w.rq.n == 0);
        }
      }
      cut(w);
    } while (!counts(w));
    return true;
  }
  // The first block of a share whose first unit is number `off` among those of request w.b (w.rq, and w.left units of the share), of which each
  // KV head has `cost`.  False if the share has nothing to do.
  template <typename F>
  OA_INLINE bool enter(Piece& w, int64_t off, int64_t cost, F request) const {
    // (a prompt of a million tokens has more than 2^32 units; the short division where it will do)
    w.h = ((uint64_t)off | (uint64_t)cost) >> 32 ? (int)(off / cost) : (int)((uint32_t)off / (uint32_t)cost);
    off -= w.h * cost;
    for (w.rb = 0;; ++w.rb) {
      const int of_block = units(block(w.rq, w.rb));
      if (off < of_block) break;
      off -= of_block;
    }
    w.off = (int)off;
    cut(w);
    return (counts(w) && !(p.uncut && w.off > 0)) || follow(w, request);
  }
};

}  // namespace omniattn
