// Blocks and shares of tree attention on the host, with the code that the kernels use (csrc/gqa_deal.h).  Reads calls from stdin, one per line,
//   rows kv_heads group S W shares batch  L_0 n_0  L_1 n_1 ...
// and checks that the shares have every unit of every block once and in order, that a block's units hold all that its queries can keep (nodes, and what the
// rule keeps of the text for a position of a node), and, where the request is short, no page without such a token.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2511_22481_amd/csrc/gqa_deal.h"

using namespace omniattn;

struct Call {
  int group, S, W, kv_heads, uncut, shares;
  std::vector<Request> requests;
};

[[noreturn]] static void wrong(const char* what, int b, int at) {
  std::printf("%s: request %d, %d\n", what, b, at);
  std::exit(1);
}

template <int R>
static void check(const Call& c) {
  const Walk<R, 2, 128, Call, true> walk(c);
  const int batch = (int)c.requests.size();
  std::vector<int64_t> begin(batch + 1, 0), cost(batch);
  for (int b = 0; b < batch; ++b) {
    const Request& r = c.requests[b];
    cost[b] = walk.cost_of(r);
    begin[b + 1] = begin[b] + cost[b] * c.kv_heads;
    for (int rb = 0; rb < blocks_of<R>(c, r); ++rb) {
      const Block k = walk.block(r, rb);
      const int grain = 128 >> tree_split<R>(c, r, rb), text = r.L - r.n;
      if (r.L > 100000) continue;
      std::vector<char> has(r.L + 129, 0);
      int last = -1;
      for (int i = 0; i < k.pages.count(); ++i) {
        const int at = k.pages.logical(i);
        if (at <= last || (int64_t)at * grain >= r.L + (int64_t)grain) wrong("a unit out of order or behind the request", b, at);
        last = at;
        bool some = false;
        for (int j = at * grain; j < (at + 1) * grain && j < r.L + 129; ++j) has[j] = 1;
        // (of the page that it lies in, as a page that holds nothing may not be there)
        const int page = at * grain / 128 * 128;
        for (int j = page; j < page + 128 && j < r.L; ++j) some |= j < c.S || j >= text || (c.W > 0 && (int64_t)j >= (int64_t)text + 1 - c.W);
        if (!some) wrong("a page of nothing", b, at);
      }
      for (int j = 0; j < r.L; ++j) {
        const bool node = j >= text && j < text + 64 && (c.W > 0 || text < c.S);
        const bool kept = j < text && (j < c.S || (c.W > 0 && (int64_t)j >= (int64_t)text + 1 - c.W));
        if ((node || kept) && !has[j]) wrong("a token is missing", b, j);
      }
    }
  }
  const Shares shares(begin[batch], c.shares);
  auto request = [&](int b) {
    if (b >= batch) wrong("past the last request", b, 0);
    return c.requests[b];
  };
  int64_t units = 0, blocks = 0, want = 0, want_blocks = 0;
  for (const Request& r : c.requests)
    for (int rb = 0; rb < blocks_of<R>(c, r); ++rb) {
      want += (int64_t)walk.block(r, rb).pages.count() * c.kv_heads;
      want_blocks += c.kv_heads;
    }
  for (int share = 0; share < shares.U; ++share) {
    const int64_t first = shares.bound(share);
    Piece w{};
    w.left = shares.bound(share + 1) - first;
    while (begin[w.b + 1] <= first) ++w.b;
    w.rq = c.requests[w.b];
    for (bool some = walk.enter(w, first - begin[w.b], cost[w.b], request); some; some = walk.follow(w, request)) {
      units += w.tile_hi - w.tile_lo;
      blocks += w.tile_lo == 0;
    }
  }
  if (units != want || blocks != want_blocks) wrong("units or blocks", (int)(units - want), (int)(blocks - want_blocks));
}

int main() {
  int rows, batch, calls = 0;
  Call c{};
  while (std::scanf("%d %d %d %d %d %d %d", &rows, &c.kv_heads, &c.group, &c.S, &c.W, &c.shares, &batch) == 7) {
    c.requests.assign((size_t)batch, Request{});
    int begin = 0;
    for (Request& r : c.requests) {
      if (std::scanf("%d %d", &r.L, &r.n) != 2) return 2;
      r.begin = begin;
      begin += r.n;
    }
    if (rows == 16) check<16>(c);
    else if (rows == 64) check<64>(c);
    else if (rows == 128) check<128>(c);
    else return 3;
    ++calls;
  }
  std::printf("ok %d\n", calls);
  return 0;
}
