// Deals out the work of grouped-query attention on the host with the code that the kernels use (csrc/gqa_deal.h), for requests of any size.
// Reads calls from stdin, one per line,
//   rows start grain kv_heads group S W uncut shares batch  L_0 n_0  L_1 n_1 ...
// and checks that the shares, one behind the other, have every page of every block of every KV head once and in order, blocks without
// pages once too, and that `owner` names the share of a block's last unit.  Prints the number of calls, or what is wrong.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2511_22481_amd/csrc/gqa_deal.h"

using namespace omniattn;

struct Call {
  int group, S, W, kv_heads, uncut, shares;
  std::vector<Request> requests;
};

[[noreturn]] static void wrong(const char* what, int share, const Piece& w) {
  std::printf("%s: share %d, request %d, head %d, block %d, unit %d, pages %d to %d\n", what, share, w.b, w.h, w.rb, w.off, w.tile_lo, w.tile_hi);
  std::exit(1);
}

// The next piece of work, as a loop over everything meets it.
struct Cursor {
  int b = 0, h = 0, rb = 0, tile = 0;
};

template <int R, int START, int GRAIN>
static void check(const Call& c) {
  const Walk<R, START, GRAIN, Call> walk(c);
  const int batch = (int)c.requests.size();
  std::vector<int64_t> cost(batch), begin(batch + 1, 0);
  for (int b = 0; b < batch; ++b) {
    cost[b] = walk.cost_of(c.requests[b]);
    begin[b + 1] = begin[b] + cost[b] * c.kv_heads;
  }
  Cursor at;
  auto settle = [&] {
    while (at.b < batch && at.rb >= blocks_of<R>(c, c.requests[at.b])) {
      at.rb = 0;
      if (c.requests[at.b].n == 0 || ++at.h == c.kv_heads) at.h = 0, ++at.b;
    }
  };
  settle();
  int share = 0;
  Piece w{};
  auto request = [&](int b) {
    if (b >= batch) wrong("past the last request", share, w);
    return c.requests[b];
  };
  const Shares shares(begin[batch], c.shares);
  if (shares.U < 0 || shares.bound(0) != 0 || shares.bound(shares.U) != begin[batch]) wrong("bounds", -1, w);
  for (; share < shares.U; ++share) {
    const int64_t first = shares.bound(share);
    w = Piece{};
    w.left = shares.bound(share + 1) - first;
    while (begin[w.b + 1] <= first) ++w.b;
    w.rq = c.requests[w.b];
    for (bool some = walk.enter(w, first - begin[w.b], cost[w.b], request); some; some = walk.follow(w, request)) {
      if (at.b >= batch || w.b != at.b || w.h != at.h || w.rb != at.rb || w.tile_lo != at.tile) wrong("not the next piece", share, w);
      const int pages = w.bk.pages.count();
      if (w.tile_hi < w.tile_lo || w.tile_hi > pages) wrong("pages", share, w);
      if (shares.owner(first) != share) wrong("owner of a share's first unit", share, w);
      at.tile = w.tile_hi;
      if (at.tile == pages) {
        // (where the block's last unit is, from what the kernel knows)
        const int64_t last = shares.bound(share + 1) - w.left - w.off + walk.units(w.bk) - 1;
        if (!c.uncut && pages > 0 && shares.owner(last) != share) wrong("owner of a block's last unit", share, w);
        at.tile = 0;
        ++at.rb;
        settle();
      }
    }
  }
  if (at.b != batch || at.tile != 0) wrong("left over", share, w);
}

int main() {
  int rows, start, grain, batch, calls = 0;
  Call c{};
  while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &rows, &start, &grain, &c.kv_heads, &c.group, &c.S, &c.W, &c.uncut, &c.shares, &batch) == 10) {
    c.requests.assign((size_t)batch, Request{});
    int begin = 0;
    for (Request& r : c.requests) {
      if (std::scanf("%d %d", &r.L, &r.n) != 2) return 2;
      r.begin = begin;
      begin += r.n;
    }
    if (rows == 16 && start == 2 && grain == 128) check<16, 2, 128>(c);
    else if (rows == 32 && start == 2 && grain == 128) check<32, 2, 128>(c);
    else if (rows == 64 && start == 2 && grain == 128) check<64, 2, 128>(c);
    else if (rows == 16 && start == 4 && grain == 32) check<16, 4, 32>(c);
    else return 3;
    ++calls;
  }
  std::printf("ok %d\n", calls);
  return 0;
}
