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
#include "cut.hpp"
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
// HBM bounds it: 94 MB in 18.6 us, 5.1 TB/s (4096 x 768 x 2048 in fp32). Planes formed
// while the products fetch them would be formed once per tile that reads them.
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
  Product q[3];
  for (int i = 0; i < a.nprob; ++i) q[i] = {a.p[i].m, a.p[i].n, a.p[i].k, a.p[i].nsrc};
  const Cut c = cut_products(q, a.nprob, EPI, F32, a.ldf);
  int64_t tiles = 0;
  for (int i = 0; i < a.nprob; ++i) {
    FfnProb &p = a.p[i];
    p.tm = int32_t(tiles_m(q[i], kTiles[c.kind]));
    p.tn = int32_t(tiles_n(q[i], kTiles[c.kind], EPI, a.ldf));
    p.tile0 = int32_t(tiles);
    tiles += int64_t(p.tm) * p.tn;
  }
  if (!tiles) return;
  a.whole = int32_t(c.whole);
  a.tail = int32_t(c.tail);
  a.slabs = int32_t(slabs_of(q[0], F32));
  a.parts = int32_t(c.parts);
  a.per = int32_t(c.per);
  // 128-tiles of which no CU has two: eight waves of 32 x 64 instead of four of 64 x 64,
  // so that each SIMD has a second wave while one waits, and a third LDS stage (us of
  // four waves and eight: 100 x 1536 x 6144 bf16 forward 39.5, 35.4; 501 x 1280 x 3456
  // forward 37.8, 35.7; 2048 x 576 x 1536 backward 73.5, 69)
  if (c.kind == 0) launch_tiles<0, 2, 4, 2, AK, BK, EPI, F32>(a, st);
  else if (c.whole + c.tail * c.parts <= kCus) launch_tiles<1, 4, 2, 3, AK, BK, EPI, F32>(a, st);
  else launch_tiles<1, 2, 2, 2, AK, BK, EPI, F32>(a, st);
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
  l.part = take(FfnProducts{s.tokens, s.dim, s.inner, s.ldf(), s.dtype == SLORR_F32}.part_bytes(bwd));
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
