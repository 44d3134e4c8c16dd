// Gated feed-forward block (see ffn_gemm.hpp for the products):
//
//   k_ffn       the products, with the activation and its backward fused into
//               their epilogues
//   k_planes    operands laid out in 16-byte rows: bf16 rows padded to a
//               multiple of 8, fp32 values as three bf16 planes
//   k_tail      the parts of tiles that were cut along k, added in order
//   k_few       the forward products for a few tokens
#include <algorithm>
#include <type_traits>

#include "block.hpp"
#include "ffn_gemm.hpp"
#include "layout.hpp"

namespace slorr {
namespace {

void check(hipError_t e, const char *what) {
  if (e != hipSuccess) throw HipError(std::string(what) + ": " + hipGetErrorString(e));
}

// rows x cols values -> bf16 rows of ld numbers, zero padded (F32: three planes).
// A call's operands go in one launch, one grid row each. Rows need no 16-byte
// alignment: the memory system takes 16-byte loads at any multiple of an element.
struct Lay {
  const void *src;
  char *dst;
  int64_t rows, lds, plane;
  int32_t cols, ld;
};
struct LayArgs {
  Lay job[5];
};
template <bool F32>
__global__ __launch_bounds__(256) void k_planes(LayArgs args) {
  using T = typename std::conditional<F32, float, uint16_t>::type;
  typedef u32x4 u32x4_any __attribute__((aligned(2)));
  Lay a = args.job[0];
#pragma unroll
  for (int i = 1; i < 5; ++i)
    if (int(blockIdx.y) == i) a = args.job[i];
  const int pieces = a.ld >> 3;
  const int64_t total = a.rows * pieces;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / pieces;
    const int c = int(i - r * pieces) * 8;
    const T *p = static_cast<const T *>(a.src) + r * a.lds + c;
    float v[8];
    if (c + 8 <= a.cols) {
      const __attribute__((address_space(1))) u32x4_any *q = (const __attribute__((address_space(1))) u32x4_any *)p;
      if constexpr (F32) {
        const u32x4 q0 = q[0], q1 = q[1];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j < 4 ? q0[j & 3] : q1[j & 3]);
      } else {
        *reinterpret_cast<u32x4 *>(a.dst + (r * a.ld + c) * 2) = q[0];
        continue;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c + j < a.cols ? to_f(p[j]) : 0.0f;
    }
    store_planes<F32>(a.dst + (r * a.ld + c) * 2, a.plane, v);
  }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The block tiles: 256 x 256 (8 waves of 128 x 64), 256 x 128 (8 of 64 x 64, three
// LDS stages) and 128 x 128 (4 of 64 x 64, two blocks per CU). Microseconds of a
// round of blocks: per slab of k with every CU at work (alone: with one block of
// the smallest per CU at most, where a slab's latency is all there is), and for
// its start and end (kActBack, which loads and stores five values per sum: back).
// From 16384 x 1536 x 6144 in bf16, us of the three tiles: the weight gradients'
// 256 slabs 467, 288 and 276 a round, y's 96 slabs 184, 118 and 119, dh's 24 slabs
// 87, 46 and 47 (a round of the first is twice the work of the others').
struct TileKind {
  int bm, bn, slots;
  double slab, alone, ends, back;
};
constexpr TileKind kTiles[] = {{256, 256, kCus, 1.77, 1.77, 13, 44},
                               {256, 128, kCus, 1.15, 1.15, 10, 20},
                               {128, 128, 2 * kCus, 1.15, 0.75, 4, 18}};
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

template <int EPI>
int64_t tiles_m(const FfnProb &p, const TileKind &k) { return cdiv(p.m, k.bm); }
template <int EPI>
int64_t tiles_n(const FfnProb &p, const TileKind &k, int64_t ldf) {
  return EPI == kStore ? cdiv(p.n, k.bn) : cdiv(ldf, EPI == kAct ? k.bn / 2 : k.bn);
}

// The least of, over the tiles: rounds of whole tiles; whole tiles as long as they
// fill rounds, the rest cut into parts.
template <int EPI, bool F32>
Cut cut_products(const FfnProb *p, int nprob, int64_t ldf) {
  Cut best;
  double least = 0;
  const int64_t slabs = cdiv(p[0].k, 64) * p[0].nsrc * (F32 ? 6 : 1);
  for (int kind = 0; kind < 3; ++kind) {
    const TileKind &k = kTiles[kind];
    // units of n slabs
    auto time = [&](int64_t units, int64_t n, double ends) {
      const int64_t full = units / k.slots, rest = units - full * k.slots;
      return double(full) * (double(n) * k.slab + ends) + (rest ? double(n) * (rest > kCus ? k.slab : k.alone) + ends : 0.0);
    };
    const double ends = EPI == kActBack ? k.back : k.ends;
    int64_t tiles = 0;
    for (int i = 0; i < nprob; ++i) tiles += tiles_m<EPI>(p[i], k) * tiles_n<EPI>(p[i], k, ldf);
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

template <int KIND, int WGM, int WGN, int NS, bool AK, bool BK, int EPI, bool F32>
void launch_tiles(const FfnArgs &a, hipStream_t st) {
  constexpr int BM = kTiles[KIND].bm, BN = kTiles[KIND].bn;
  const dim3 grid(uint32_t(a.whole + a.tail * a.parts));
  hipLaunchKernelGGL((k_ffn<BM, BN, WGM, WGN, NS, AK, BK, EPI, F32>), grid, dim3(64 * WGM * WGN), 0, st, a);
  check(hipGetLastError(), "kernel launch");
  if (!a.tail) return;
  const dim3 pieces(uint32_t(BM * BN / (EPI == kAct ? 16 : 8) / 256), uint32_t(a.tail));
  hipLaunchKernelGGL((k_tail<BM, BN, EPI, F32>), pieces, dim3(256), 0, st, a);
  check(hipGetLastError(), "kernel launch");
}

template <bool AK, bool BK, int EPI, bool F32>
void launch_products(FfnArgs &a, hipStream_t st) {
  const Cut c = cut_products<EPI, F32>(a.p, a.nprob, a.ldf);
  int64_t tiles = 0;
  for (int i = 0; i < a.nprob; ++i) {
    FfnProb &p = a.p[i];
    p.tm = int32_t(tiles_m<EPI>(p, kTiles[c.kind]));
    p.tn = int32_t(tiles_n<EPI>(p, kTiles[c.kind], a.ldf));
    p.tile0 = int32_t(tiles);
    tiles += int64_t(p.tm) * p.tn;
  }
  if (!tiles) return;
  a.whole = int32_t(c.whole);
  a.tail = int32_t(c.tail);
  a.slabs = int32_t(cdiv(a.p[0].k, 64)) * a.p[0].nsrc * (F32 ? 6 : 1);
  a.parts = int32_t(c.parts);
  a.per = int32_t(c.per);
  if (c.kind == 0) launch_tiles<0, 2, 4, 2, AK, BK, EPI, F32>(a, st);
  else if (c.kind == 1) launch_tiles<1, 4, 2, 3, AK, BK, EPI, F32>(a, st);
  else launch_tiles<2, 2, 2, 2, AK, BK, EPI, F32>(a, st);
}

// The state's parts: a, b, and in bf16 their exponents (16 bytes per row and 128
// columns).
size_t exponents(const FfnShape &s) {
  return s.dtype == SLORR_BF16 ? size_t(cdiv(s.ldf(), 128)) * size_t(s.tokens) * 16 : 0;
}
void state_parts(const FfnShape &s, void *state, FfnArgs &a) {
  if (!state) return;
  const size_t n = size_t(s.tokens) * size_t(s.ldf()) * s.elem();
  char *p = static_cast<char *>(state);
  uint8_t *e = reinterpret_cast<uint8_t *>(p) + 2 * n;
  a.a = {p, e, s.tokens, int32_t(s.ldf())};
  a.b = {p + n, e + exponents(s), s.tokens, int32_t(s.ldf())};
}

// An operand as the products read it.
struct Operand {
  const char *p;
  int64_t ld, plane;
};

// The operands of a call, laid out in one launch.
template <bool F32>
struct Layer {
  const FfnShape &s;
  char *ws;
  LayArgs args{};
  int n = 0;
  int64_t most = 0;
  Operand add(const void *src, int64_t rows, int32_t cols, int64_t lds, size_t off) {
    if (off == kAbsent) return {static_cast<const char *>(src), lds, 0};
    const Operand o{ws + off, up8(cols), rows * up8(cols) * 2};
    if (rows) {
      args.job[n++] = {src, ws + off, rows, lds, o.plane, cols, int32_t(o.ld)};
      most = std::max(most, rows * (o.ld / 8));
    }
    return o;
  }
  void run(hipStream_t st) const {
    if (!n) return;
    const dim3 grid(uint32_t(std::min<int64_t>(cdiv(most, 256), 8 * kCus)), uint32_t(n));
    hipLaunchKernelGGL(k_planes<F32>, grid, dim3(256), 0, st, args);
    check(hipGetLastError(), "kernel launch");
  }
};

FfnProb product(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, void *out, int64_t ldo) {
  FfnProb p{};
  p.a[0] = a.p;
  p.b[0] = b.p;
  p.pa = a.plane;
  p.pb = b.plane;
  p.lda = a.ld;
  p.ldb = b.ld;
  p.m = int32_t(m);
  p.n = int32_t(n);
  p.k = int32_t(k);
  p.nsrc = 1;
  p.out = out;
  p.ldo = ldo;
  return p;
}

template <bool DUAL, bool F32>
void launch_few(const FewArgs &a, hipStream_t st) {
  // waves: at least two chunks of k each
  const int chunks = int(cdiv(a.k, F32 ? 32 : 64)), most = a.tokens > 32 ? 8 : 16;
  int waves = 4;
  while (waves < most && chunks >= 4 * waves) waves *= 2;
  const dim3 grid(uint32_t(cdiv(a.n, 16))), block(64 * waves);
  if (a.tokens > 32) hipLaunchKernelGGL((k_few<4, DUAL, F32>), grid, block, 0, st, a);
  else if (a.tokens > 16) hipLaunchKernelGGL((k_few<2, DUAL, F32>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_few<1, DUAL, F32>), grid, block, 0, st, a);
  check(hipGetLastError(), "kernel launch");
}

template <bool F32>
void forward(const FfnShape &s, const void *x, const void *wg, const void *wu, const void *wd, void *y, void *state,
             char *ws, hipStream_t st) {
  const FfnLayout l = ffn_layout(s, false);
  const int64_t T = s.tokens;
  if (s.few() && !state) {
    launch_few<true, F32>({x, wg, wu, ws, s.ldx, s.ldf(), int32_t(T), s.inner, s.dim, s.act}, st);
    launch_few<false, F32>({ws, wd, nullptr, y, s.ldf(), s.dim, int32_t(T), s.dim, s.inner, s.act}, st);
    return;
  }
  Layer<F32> lay{s, ws};
  const Operand X = lay.add(x, T, s.dim, s.ldx, l.x);
  const Operand G = lay.add(wg, s.inner, s.dim, s.dim, l.wg);
  const Operand U = lay.add(wu, s.inner, s.dim, s.dim, l.wu);
  const Operand D = lay.add(wd, s.dim, s.inner, s.inner, l.wd);
  lay.run(st);
  const Operand H{ws + l.h, s.ldf(), T * s.ldf() * 2};
  FfnArgs a{};
  a.nprob = 1;
  a.act = s.act;
  a.ldf = int32_t(s.ldf());
  a.part = reinterpret_cast<float *>(ws + l.part);
  a.p[0] = product(X, G, T, s.inner, s.dim, nullptr, 0);
  a.p[0].b[1] = U.p;
  state_parts(s, state, a);
  a.h = ws + l.h;
  a.plane = H.plane;
  launch_products<false, false, kAct, F32>(a, st);
  a.p[0] = product(H, D, T, s.dim, s.inner, y, s.dim);
  launch_products<false, false, kStore, F32>(a, st);
}

template <bool F32>
void backward(const FfnShape &s, const void *dy, const void *x, const void *wg, const void *wu, const void *wd,
              const void *state, void *dx, void *dwg, void *dwu, void *dwd, char *ws, hipStream_t st) {
  const FfnLayout l = ffn_layout(s, true);
  const int64_t T = s.tokens;
  const bool by_x = dwg || dwu;
  Layer<F32> lay{s, ws};
  Operand D{}, G{}, U{}, X{};
  const Operand DY = lay.add(dy, T, s.dim, s.lddy, l.dy);
  if (T) D = lay.add(wd, s.dim, s.inner, s.inner, l.wd);
  if (T && dx) {
    G = lay.add(wg, s.inner, s.dim, s.dim, l.wg);
    U = lay.add(wu, s.inner, s.dim, s.dim, l.wu);
  }
  if (by_x) X = lay.add(x, T, s.dim, s.ldx, l.x);
  lay.run(st);
  const int64_t plane = T * s.ldf() * 2;
  const Operand H{ws + l.h, s.ldf(), plane}, DA{ws + l.da, s.ldf(), plane}, DB{ws + l.db, s.ldf(), plane};
  FfnArgs a{};
  a.act = s.act;
  a.ldf = int32_t(s.ldf());
  a.part = reinterpret_cast<float *>(ws + l.part);
  if (T) {
    a.nprob = 1;
    a.p[0] = product(DY, D, T, s.inner, s.dim, nullptr, 0);
    state_parts(s, const_cast<void *>(state), a);
    a.h = ws + l.h;
    a.da = ws + l.da;
    a.db = ws + l.db;
    a.plane = plane;
    launch_products<false, true, kActBack, F32>(a, st);
  }
  if (dx && T) {
    a.nprob = 1;
    a.p[0] = product(DA, G, T, s.dim, s.inner, dx, s.dim);
    a.p[0].a[1] = DB.p;
    a.p[0].b[1] = U.p;
    a.p[0].nsrc = 2;
    launch_products<false, true, kStore, F32>(a, st);
  }
  if (dwg || dwu || dwd) {
    a.nprob = 0;
    if (dwg) a.p[a.nprob++] = product(DA, X, s.inner, s.dim, T, dwg, s.dim);
    if (dwu) a.p[a.nprob++] = product(DB, X, s.inner, s.dim, T, dwu, s.dim);
    if (dwd) a.p[a.nprob++] = product(DY, H, s.dim, s.inner, T, dwd, s.inner);
    launch_products<true, true, kStore, F32>(a, st);
  }
}

}  // namespace

FfnLayout ffn_layout(const FfnShape &s, bool bwd) {
  FfnLayout l;
  const size_t pl = size_t(s.planes()) * 2;
  auto take = [&](size_t bytes) {
    const size_t at = l.bytes;
    l.bytes += (bytes + 255) & ~size_t(255);
    return at;
  };
  const size_t T = size_t(s.tokens), w = size_t(s.inner) * size_t(s.ldd()) * pl;
  if (!s.direct(s.dim, s.ldx)) l.x = take(T * size_t(s.ldd()) * pl);
  if (bwd && !s.direct(s.dim, s.lddy)) l.dy = take(T * size_t(s.ldd()) * pl);
  if (!s.direct(s.dim, s.dim)) {
    l.wg = take(w);
    l.wu = take(w);
  }
  if (!s.direct(s.inner, s.inner)) l.wd = take(size_t(s.dim) * size_t(s.ldf()) * pl);
  l.h = take(T * size_t(s.ldf()) * pl);
  if (bwd) {
    l.da = take(T * size_t(s.ldf()) * pl);
    l.db = take(T * size_t(s.ldf()) * pl);
  }
  // parts of cut tiles: what the launches of the call need at most (the weight
  // gradients that are asked for are a launch: `same` of inner x dim, `other` of
  // dim x inner)
  const bool f32 = s.dtype == SLORR_F32;
  auto need = [&](auto epi, int same, int other, int64_t m, int64_t n, int64_t k, int nsrc) {
    constexpr int EPI = decltype(epi)::value;
    FfnProb p[3]{};
    for (int i = 0; i < same + other; ++i) {
      p[i].m = int32_t(i < same ? m : n);
      p[i].n = int32_t(i < same ? n : m);
      p[i].k = int32_t(k);
      p[i].nsrc = nsrc;
    }
    const int nprob = same + other;
    const Cut c = f32 ? cut_products<EPI, true>(p, nprob, s.ldf()) : cut_products<EPI, false>(p, nprob, s.ldf());
    return c.part_bytes();
  };
  std::integral_constant<int, kStore> store;
  size_t part = 0;
  if (!bwd) {
    part = std::max(need(std::integral_constant<int, kAct>{}, 1, 0, s.tokens, s.inner, s.dim, 1),
                    need(store, 1, 0, s.tokens, s.dim, s.inner, 1));
  } else {
    part = std::max(need(std::integral_constant<int, kActBack>{}, 1, 0, s.tokens, s.inner, s.dim, 1),
                    need(store, 1, 0, s.tokens, s.dim, s.inner, 2));
    for (int same = 0; same <= 2; ++same)
      for (int other = 0; other <= 1; ++other)
        if (same + other) part = std::max(part, need(store, same, other, s.inner, s.dim, s.tokens, 1));
  }
  l.part = take(part);
  l.bytes = std::max(l.bytes, size_t(256));
  return l;
}

size_t ffn_state_bytes(const FfnShape &s) {
  return std::max(size_t(256), 2 * (size_t(s.tokens) * size_t(s.ldf()) * s.elem() + exponents(s)));
}

void enqueue_ffn_forward(const FfnShape &s, const void *x, const void *wg, const void *wu, const void *wd, void *y,
                         void *state, void *ws, hipStream_t st) {
  if (!s.tokens) return;
  if (s.dtype == SLORR_F32) forward<true>(s, x, wg, wu, wd, y, state, static_cast<char *>(ws), st);
  else forward<false>(s, x, wg, wu, wd, y, state, static_cast<char *>(ws), st);
}

void enqueue_ffn_backward(const FfnShape &s, const void *dy, const void *x, const void *wg, const void *wu,
                          const void *wd, const void *state, void *dx, void *dwg, void *dwu, void *dwd, void *ws,
                          hipStream_t st) {
  if (s.dtype == SLORR_F32) backward<true>(s, dy, x, wg, wu, wd, state, dx, dwg, dwu, dwd, static_cast<char *>(ws), st);
  else backward<false>(s, dy, x, wg, wu, wd, state, dx, dwg, dwu, dwd, static_cast<char *>(ws), st);
}

}  // namespace slorr
