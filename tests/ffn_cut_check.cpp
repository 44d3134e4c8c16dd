// How the feed-forward's launches are cut into blocks (csrc/cut.hpp), on the CPU:
// for every launch of a call, every slab of k of every tile belongs to one block,
// tiles cover their products once, no part is empty, and the parts' sums lie
// apart and inside the room that the call's workspace keeps for them. Input
// (stdin): lines of tokens dim inner f32; built by tests/test_block_cut.py.
#include <cstdio>
#include <iostream>
#include <set>
#include <utility>
#include <vector>

#include "cut.hpp"

using namespace slorr;

static int bad = 0;
static long launches = 0, cut = 0, kinds[2] = {};

static void fail(const char *m, int64_t a, int64_t b) {
  if (++bad < 20) std::printf("FAIL %s: %lld %lld\n", m, (long long)a, (long long)b);
}

static void launch(const Cut &c, const std::vector<Product> &p, int epi, bool f32, int64_t ldf, size_t room) {
  ++launches;
  if (c.kind < 0 || c.kind > 1) return fail("kind", c.kind, 0);
  ++kinds[c.kind];
  cut += c.tail > 0;
  const TileKind &k = kTiles[c.kind];
  int64_t tiles = 0;
  for (const Product &q : p) {
    const int tm = int(tiles_m(q, k)), tn = int(tiles_n(q, k, epi, ldf));
    const int width = epi == kAct ? k.bn / 2 : k.bn;
    const int64_t cols = epi == kStore ? q.n : ldf;
    if (int64_t(tm) * k.bm < q.m || int64_t(tn) * width < cols) fail("products are covered", tm, tn);
    if (tm && (int64_t(tm - 1) * k.bm >= q.m || int64_t(tn - 1) * width >= cols)) fail("tiles without work", tm, tn);
    std::vector<char> seen(size_t(tm) * size_t(tn));
    for (int t = 0; t < tm * tn; ++t) {
      int row = -1, col = -1;
      tile_place(t, tm, tn, row, col);
      if (row < 0 || row >= tm || col < 0 || col >= tn) { fail("tile place", row, col); continue; }
      if (seen[size_t(row) * tn + col]++) fail("tile twice", row, col);
    }
    tiles += int64_t(tm) * tn;
  }
  const int64_t slabs = slabs_of(p[0], f32);
  for (const Product &q : p)
    if (slabs_of(q, f32) != slabs) fail("products of one launch have one k", slabs, slabs_of(q, f32));
  if (c.whole + c.tail != tiles) fail("tiles", c.whole + c.tail, tiles);
  if (c.tail && c.whole % 8) fail("whole tiles keep the XCDs in turn", c.whole, 0);
  const std::vector<char> none(static_cast<size_t>(slabs));
  std::vector<std::vector<char>> done(static_cast<size_t>(tiles), none);
  std::set<int> slots;
  for (int64_t b = 0; b < c.whole + c.tail * c.parts; ++b) {
    int tile = 0, s0 = 0, s1 = int(slabs);
    if (b >= c.whole) {
      const int slot = by_xcd(int(b - c.whole), int(c.tail * c.parts));
      if (slot < 0 || slot >= c.tail * c.parts || !slots.insert(slot).second) fail("slot", slot, b);
      if (size_t(slot + 1) * size_t(k.bm) * size_t(k.bn) * 4 > room) fail("room for parts", slot, int64_t(room));
      part_place(slot, int(c.tail), int(c.per), int(slabs), tile, s0, s1);
      tile += int(c.whole);
      // k_tail's order: part q of tail tile t is slot q * tail + t
      if (slot != s0 / c.per * c.tail + tile - c.whole) fail("part order", slot, tile);
      if (s0 >= s1) fail("empty part", s0, s1);
    } else {
      tile = by_xcd(int(b), int(c.whole));
    }
    if (tile < 0 || tile >= tiles) { fail("tile", tile, tiles); continue; }
    for (int s = s0; s < s1; ++s)
      if (s < 0 || s >= slabs || done[size_t(tile)][size_t(s)]++) fail("slab", tile, s);
  }
  for (size_t t = 0; t < done.size(); ++t)
    for (size_t s = 0; s < done[t].size(); ++s)
      if (done[t][s] != 1) fail("slab not done", int64_t(t), int64_t(s));
}

int main() {
  long long t, d, n, f;
  while (std::cin >> t >> d >> n >> f) {
    const int64_t ldf = (n + 7) & ~7ll;
    const bool f32 = f != 0;
    const FfnProducts q{t, d, n, ldf, f32};
    const int before = bad;
    launch(q.act(), {{t, n, d, 1}}, kAct, f32, ldf, q.part_bytes(false));
    launch(q.y(), {{t, d, n, 1}}, kStore, f32, ldf, q.part_bytes(false));
    launch(q.dh(), {{t, n, d, 1}}, kActBack, f32, ldf, q.part_bytes(true));
    launch(q.dx(), {{t, d, n, 2}}, kStore, f32, ldf, q.part_bytes(true));
    for (int same = 0; same <= 2; ++same)
      for (int other = 0; other <= 1; ++other) {
        std::vector<Product> p;
        for (int i = 0; i < same; ++i) p.push_back({n, d, t, 1});
        for (int i = 0; i < other; ++i) p.push_back({d, n, t, 1});
        if (!p.empty()) launch(q.weights(same, other), p, kStore, f32, ldf, q.part_bytes(true));
      }
    if (bad != before) std::printf("at %lld %lld %lld %lld\n", t, d, n, f);
  }
  std::printf("%s launches=%ld cut=%ld kinds=%ld,%ld\n", bad ? "BAD" : "OK", launches, cut, kinds[0], kinds[1]);
  return bad != 0;
}
