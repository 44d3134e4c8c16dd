// How a launch of the feed-forward's products is cut into blocks, and which block
// does which part (host and device code; compiles without HIP).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "layout.hpp"

#if defined(__HIPCC__)
#define SLORR_HD __host__ __device__
#else
#define SLORR_HD
#endif

namespace slorr {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What becomes of a product's sums (see ffn_gemm.hpp).
enum FfnEpi { kStore = 0, kAct = 1, kActBack = 2 };

// The block tiles: 256 x 256 (8 waves of 128 x 64) and 128 x 128 (4 of 64 x 64, two
// blocks per CU; 8 of 32 x 64 where there is one). Microseconds of a round of
// blocks: per slab of k with every CU at work (alone: with one block per CU at most,
// where a slab's latency is all there is), and for its start and end (kActBack,
// which loads and stores five values per sum: back). From 16384 x 1536 x 6144 in
// bf16, us of a round of each: the weight gradients' 256 slabs 467 and 276, y's 96
// slabs 184 and 119, dh's 24 slabs 81 and 49 (a round of the first is twice the work
// of the other's).
// Not kept: 256 x 128 with three LDS stages (1.15 us a slab: two 128-tiles, with
// longer ends), 128 x 128 with four stages and one block per CU (0.6 us a slab:
// 16384 x 1280 x 3456 backward 1017 -> 1303 us where it ran, 100 x 1536 x 6144
// forward 40.5 -> 36.9).
struct TileKind {
  int bm, bn, slots;
  double slab, alone, ends, back;
};
constexpr TileKind kTiles[] = {{256, 256, kCus, 1.77, 1.77, 13, 38},
                               {128, 128, 2 * kCus, 1.15, 0.75, 4, 20}};
constexpr double kPartByte = 2 / 4.5e6;                   // a part's sums, written and read once at 4.5 TB/s
constexpr double kTailLaunch = 5;

// How a launch's products are cut: the tile, how many of them whole, and the
// parts of the others.
struct Cut {
  int kind = -1;
  int64_t whole = 0, tail = 0, parts = 0, per = 0;
  size_t part_bytes() const {
    return kind < 0 ? 0 : size_t(tail * parts) * size_t(kTiles[kind].bm) * size_t(kTiles[kind].bn) * 4;
  }
};

// A product C (m x n), summed over k of nsrc sources.
struct Product {
  int64_t m, n, k;
  int32_t nsrc;
};
inline int64_t slabs_of(const Product &p, bool f32) { return cdiv(p.k, 64) * p.nsrc * (f32 ? 6 : 1); }
inline int64_t tiles_m(const Product &p, const TileKind &k) { return cdiv(p.m, k.bm); }
// (kAct: a tile's columns are half a's and half b's; inner tensors' rows end at ldf)
inline int64_t tiles_n(const Product &p, const TileKind &k, int epi, int64_t ldf) {
  return epi == kStore ? cdiv(p.n, k.bn) : cdiv(ldf, epi == kAct ? k.bn / 2 : k.bn);
}

// The least of, over the tiles: rounds of whole tiles; whole tiles as long as they
// fill rounds, the rest cut into parts.
inline Cut cut_products(const Product *p, int nprob, int epi, bool f32, int64_t ldf) {
  Cut best;
  double least = 0;
  const int64_t slabs = slabs_of(p[0], f32);
  for (int kind = 0; kind < 2; ++kind) {
    const TileKind &k = kTiles[kind];
    // units of n slabs
    auto time = [&](int64_t units, int64_t n, double ends) {
      const int64_t full = units / k.slots, rest = units - full * k.slots;
      return double(full) * (double(n) * k.slab + ends) + (rest ? double(n) * (rest > kCus ? k.slab : k.alone) + ends : 0.0);
    };
    const double ends = epi == kActBack ? k.back : k.ends;
    int64_t tiles = 0;
    for (int i = 0; i < nprob; ++i) tiles += tiles_m(p[i], k) * tiles_n(p[i], k, epi, ldf);
    auto offer = [&](const Cut &c, double t) {
      if (best.kind < 0 || t < least) {
        best = c;
        least = t;
      }
    };
    Cut c;
    c.kind = kind;
    c.whole = tiles;
    offer(c, time(tiles, slabs, ends));
    c.whole = tiles / k.slots * k.slots;
    c.tail = tiles - c.whole;
    // parts of at least 4 slabs: below, a block's start and its part's way through
    // memory cost more than the slabs
    for (c.parts = 2; c.tail && c.parts <= 16 && cdiv(slabs, c.parts) >= 4; ++c.parts) {
      c.per = cdiv(slabs, c.parts);
      if (c.per * (c.parts - 1) >= slabs) continue;       // (the last part would be empty)
      offer(c, time(c.whole, slabs, ends) + time(c.tail * c.parts, c.per, k.ends) + kTailLaunch +
                   double(c.part_bytes()) * kPartByte);
    }
  }
  return best;
}

// The products of a call's launches. Forward: a and b, then y. Backward: dh; dx;
// and the weight gradients that are asked for, one launch of `same` products
// inner x dim and `other` dim x inner.
struct FfnProducts {
  int64_t tokens, dim, inner, ldf;
  bool f32;
  Cut act() const { return one({tokens, inner, dim, 1}, kAct); }
  Cut y() const { return one({tokens, dim, inner, 1}, kStore); }
  Cut dh() const { return one({tokens, inner, dim, 1}, kActBack); }
  Cut dx() const { return one({tokens, dim, inner, 2}, kStore); }
  Cut weights(int same, int other) const {
    Product p[3];
    for (int i = 0; i < same + other; ++i) {
      const bool s = i < same;
      p[i] = {s ? inner : dim, s ? dim : inner, tokens, 1};
    }
    return cut_products(p, same + other, kStore, f32, ldf);
  }
  // bytes of the parts that a call needs room for
  size_t part_bytes(bool backward) const {
    size_t b = 0;
    auto most = [&](const Cut &c) { b = c.part_bytes() > b ? c.part_bytes() : b; };
    if (!backward) {
      most(act());
      most(y());
      return b;
    }
    most(dh());
    most(dx());
    for (int same = 0; same <= 2; ++same)
      for (int other = 0; other <= 1; ++other)
        if (same + other) most(weights(same, other));
    return b;
  }

 private:
  Cut one(const Product &p, int epi) const { return cut_products(&p, 1, epi, f32, ldf); }
};

// Block b of n, consecutive ones on one XCD (block index modulo 8).
SLORR_HD inline int by_xcd(int b, int n) {
  const int xcd = b & 7, per = n >> 3, rem = n & 7;
  return xcd * per + (xcd < rem ? xcd : rem) + (b >> 3);
}

// The place of tile t of tm x tn: 8 tiles of a column of tiles follow each other.
SLORR_HD inline void tile_place(int t, int tm, int tn, int &row, int &col) {
  const int g = t / (8 * tn), r = t - g * 8 * tn, rows = tm - 8 * g < 8 ? tm - 8 * g : 8;
  col = r / rows;
  row = 8 * g + r - col * rows;
}

// The part of a tail tile in slot `slot` of `tail` x `parts`: tile `tile` of the
// tail, slabs [s0, s1).
SLORR_HD inline void part_place(int slot, int tail, int per, int slabs, int &tile, int &s0, int &s1) {
  const int q = slot / tail;
  tile = slot - q * tail;
  s0 = q * per;
  s1 = s0 + per < slabs ? s0 + per : slabs;
}

}  // namespace slorr
