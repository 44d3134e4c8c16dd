// The join between two blocks and dropout (streaming kernels):
//
//   k_join_fwd  u = N(f) w1 + b1, y = x + alpha s g D u, z = N(y) w2 + b2
//   k_join_bwd  their gradients, and per block the fp32 partial sums of the
//               vectors' gradients
//   k_join_sum  those partials added in order
//   k_dropout   y = D x
//
// N(t) = (t - mu) r with r = (mean((t - mu)^2) + eps)^-1/2; RMS: mu = 0.
// D is 0 or 1 / (1 - p') by the counter-based generator (see slorr_dropout in
// slorr.h): a 16-bit number per element, so one Philox block serves the 8
// elements of a thread's 16 bytes.
//
// Backward, with t^ the normalised row: N's input gradient is
// r (A - mean(A) - t^ mean(A t^)), A the gradient of t^ (RMS: no mean(A)).
// dY = dy + N'(dz w2); dx = dY; du = dY alpha s g D; df = N'(du w1), and the
// vectors' gradients are column sums. Nothing is kept from the forward pass: a
// row of x and f gives u, y and both norms again, and reading them costs what
// reading y and saved statistics would.
#include <algorithm>
#include <type_traits>

#include "block.hpp"
#include "cut.hpp"
#include "device.hpp"
#include "layout.hpp"

namespace slorr {
namespace {

void check(hipError_t e, const char *what) {
  if (e != hipSuccess) throw HipError(std::string(what) + ": " + hipGetErrorString(e));
}

// ------------------------------------------------------------------ generator

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);       // (the table of a ^ b ^ c)
}
// One block of Philox4x32-10: ten rounds of two 32 x 32 -> 64 products.
__device__ __forceinline__ void philox(uint64_t index, uint64_t offset, uint64_t key, uint32_t (&c)[4]) {
  c[0] = uint32_t(index);
  c[1] = uint32_t(index >> 32);
  c[2] = uint32_t(offset);
  c[3] = uint32_t(offset >> 32);
  uint32_t k0 = uint32_t(key), k1 = uint32_t(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = uint64_t(c[0]) * 0xD2511F53u, b = uint64_t(c[2]) * 0xCD9E8D57u;
    c[0] = xor3(uint32_t(b >> 32), c[1], k0);
    c[1] = uint32_t(b);
    c[2] = xor3(uint32_t(a >> 32), c[3], k1);
    c[3] = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

struct Rng {
  uint64_t key, offset;
};
__device__ __forceinline__ Rng load_rng(const int64_t *rng, int64_t site) {
  return {uint64_t(rng[0]), uint64_t(rng[1]) + uint64_t(site)};
}

// Eight elements' factors, k where element e + j is kept and 0 elsewhere. drop16
// is the threshold in the upper half of a word: the upper 16-bit number of a word
// is compared in place, the lower one shifted up. A run of eight that does not
// start at a multiple of 8 takes two generator blocks; s, the element's place in
// its block, is the same over a wave.
template <bool NOW>
__device__ __forceinline__ void keep8(int64_t e, int s, Rng r, uint32_t drop16, float k, float (&m)[8]) {
  // NOW: the rounds' keys are formed here. Held over the loop over rows they fill the
  // scalar registers and are fetched from lanes of vector ones, 29 instructions a row.
  if constexpr (NOW) asm volatile("" : "+s"(r.key));
  uint32_t c[4];
  philox(uint64_t(e) >> 3, r.offset, r.key, c);
  if (s) {
    uint32_t n[4];
    philox((uint64_t(e) >> 3) + 1, r.offset, r.key, n);
    // the eight numbers from s on: four words first, then 16 bits at a time
    const bool far = s & 4;
    const uint64_t q0 = uint64_t(c[1]) << 32 | c[0], q1 = uint64_t(c[3]) << 32 | c[2];
    const uint64_t q2 = uint64_t(n[1]) << 32 | n[0], q3 = uint64_t(n[3]) << 32 | n[2];
    const uint64_t a0 = far ? q1 : q0, a1 = far ? q2 : q1, a2 = far ? q3 : q2;
    const int b = 16 * (s & 3);
    const uint64_t t0 = b ? a0 >> b | a1 << (64 - b) : a0, t1 = b ? a1 >> b | a2 << (64 - b) : a1;
    c[0] = uint32_t(t0);
    c[1] = uint32_t(t0 >> 32);
    c[2] = uint32_t(t1);
    c[3] = uint32_t(t1 >> 32);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[2 * i] = c[i] << 16 >= drop16 ? k : 0.0f;
    m[2 * i + 1] = c[i] >= drop16 ? k : 0.0f;
  }
}

// ------------------------------------------------------------------- accesses

template <typename T>
__device__ __forceinline__ void put(T *row, int c, int dim, const float (&v)[8]) {
  Raw<T> r;
  if constexpr (sizeof(T) == 2) {
    typedef float floatx8 __attribute__((ext_vector_type(8)));
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    floatx8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = v[j];
    r.q[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.q[j >> 2][j & 3] = __float_as_uint(v[j]);
  }
  if (c + 8 <= dim) {
    SLORR_GLOBAL u32x4_any *p = (SLORR_GLOBAL u32x4_any *)(row + c);
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) p[i] = r.q[i];
    return;
  }
  const int n = dim - c;
  if (n <= 0) return;
  const bool h4 = n & 4, h2 = n & 2;
  T *p2 = row + c + (n & 4), *p1 = row + c + (n & 6);
  if constexpr (sizeof(T) == 2) {
    const uint32_t lo = h4 ? r.q[0][2] : r.q[0][0], hi = h4 ? r.q[0][3] : r.q[0][1];
    if (h4) *(SLORR_GLOBAL u32x2_any *)(row + c) = u32x2_any{r.q[0][0], r.q[0][1]};
    if (h2) *(SLORR_GLOBAL u32_any *)p2 = lo;
    if (n & 1) *(SLORR_GLOBAL uint16_t *)p1 = uint16_t(h2 ? hi : lo);
  } else {
    const u32x4 e = h4 ? r.q[sizeof(T) / 2 - 1] : r.q[0];
    if (h4) *(SLORR_GLOBAL u32x4_any *)(row + c) = r.q[0];
    if (h2) *(SLORR_GLOBAL u32x2_any *)p2 = u32x2_any{e[0], e[1]};
    if (n & 1) *(SLORR_GLOBAL u32_any *)p1 = h2 ? e[2] : e[0];
  }
}

// A row's piece. WHOLE: rows of whole pieces (dim a multiple of 8), without the code
// for a row's last columns.
template <bool WHOLE, typename T>
__device__ __forceinline__ Raw<T> piece_of(const T *row, int c, int dim) {
  if constexpr (!WHOLE) return get(row, c, dim);
  Raw<T> r = {};
  if (c < dim) {
    const SLORR_GLOBAL u32x4_any *p = (const SLORR_GLOBAL u32x4_any *)(row + c);
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) r.q[i] = p[i];
  }
  return r;
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void put_piece(T *row, int c, int dim, const float (&v)[8]) {
  if constexpr (!WHOLE) put(row, c, dim, v);
  else if (c < dim) put(row + c, 0, 8, v);
}

// NV pieces of 8 columns per thread, as fp32.
template <int NV>
struct Row {
  float v[NV][8];
};
__device__ __forceinline__ int column(int v) { return (v * int(blockDim.x) + int(threadIdx.x)) * 8; }

template <typename T, bool WHOLE>
__device__ __forceinline__ void vector8(const void *p, int c, int dim, float none, float (&o)[8]) {
  if (p) {
    widen<T>(piece_of<WHOLE>(static_cast<const T *>(p), c, dim), o);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = none;
  }
}

// The sum over a wave, in every lane: within a row of 16 lanes by data-parallel
// moves, then across rows by the lane swaps.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_total(float v) {
  v += dpp<0xB1>(v);                       // quad_perm [1, 0, 3, 2]
  v += dpp<0x4E>(v);                       // quad_perm [2, 3, 0, 1]
  v += dpp<0x141>(v);                      // row_half_mirror
  v += dpp<0x140>(v);                      // row_mirror
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sums over the block, the result in every thread: each wave's total, then the
// waves' in order. Two buffers, used in turn: a wave that writes one again has
// passed the barrier after the other's reads. Entries of waves that the block
// does not have hold zeros.
struct RowSums {
  float v[2][2][8];
};
__device__ __forceinline__ void row_sums_init(RowSums &sh) {
  if (threadIdx.x < 32) (&sh.v[0][0][0])[threadIdx.x] = 0.0f;
  __syncthreads();
}
template <int K>
__device__ __forceinline__ void row_sum(float (&p)[K], RowSums &sh, int &turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) p[k] = wave_total(p[k]);
  if (blockDim.x == 64) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) sh.v[turn][k][threadIdx.x >> 6] = p[k];
  __syncthreads();
  const float4v *s = reinterpret_cast<const float4v *>(&sh.v[turn][0][0]);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const float4v a = s[2 * k], b = s[2 * k + 1];
    p[k] = ((a[0] + a[1]) + (a[2] + a[3])) + ((b[0] + b[1]) + (b[2] + b[3]));
  }
  turn ^= 1;
}

struct JoinArgs {
  const void *x, *f, *w1, *b1, *gate, *scale, *w2, *b2;
  const int64_t *rng;
  void *y, *z;                                  // forward
  const void *dy, *dz;                          // backward
  void *dx, *df, *dgate;
  float *part;                                  // [5][blocks][ldp]: w1, b1, scale, w2, b2; null: none wanted
  float *gpart;                                 // [blocks][ldp]; null: dgate is written directly
  int64_t rows, ldx, ldf, ldg, gate_rows, gate_run;   // gate_run: rows per gate row
  int64_t per_block;                            // forward: rows per block
  int64_t groups, rpg, gpb, parts, rpp;         // JoinCut
  int64_t site;
  int32_t dim, ldp, layer, post, pre;
  uint32_t drop16;                              // threshold in a word's upper half; 0: keep all
  float eps, inv, k;                            // inv: 1 / dim; k: alpha / (1 - p')
};

// t - mu in place; columns past dim become zero.
template <int NV>
__device__ __forceinline__ void subtract_mean(Row<NV> &t, float mu, int dim) {
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) t.v[v][j] = column(v) + j < dim ? t.v[v][j] - mu : 0.0f;
}

// mu out of t, and r of the norm; t^ is r t.
template <int NV>
__device__ __forceinline__ float norm_of(Row<NV> &t, const JoinArgs &a, RowSums &sh, int &turn) {
  float p[1];
  if (a.layer) {
    p[0] = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) p[0] += t.v[v][j];
    row_sum<1>(p, sh, turn);
    subtract_mean(t, p[0] * a.inv, a.dim);
  }
  p[0] = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) p[0] = fmaf(t.v[v][j], t.v[v][j], p[0]);
  row_sum<1>(p, sh, turn);
  return __builtin_amdgcn_rsqf(fmaf(p[0], a.inv, a.eps));
}

// The factors of a row's piece: k D.
template <bool NOW>
__device__ __forceinline__ void factors(const JoinArgs &a, const Rng &rng, int64_t row, int c, float k, float (&m)[8]) {
  if (a.drop16) {
    const int64_t base = row * a.dim;
    keep8<NOW>(base + c, int(base) & 7, rng, a.drop16, k, m);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = k;
  }
}

// A pointer whose loads are not moved: left to itself the compiler reads the
// vectors once and holds them in registers over the loop over rows.
__device__ __forceinline__ const void *unmoved(const void *p) {
  asm volatile("" : "+s"(p));
  return p;
}

// s g w1 and s g b1 of a piece for a gate row (null: 1).
template <typename T, bool WHOLE>
__device__ __forceinline__ void product8(const JoinArgs &a, const T *gate, int v, float (&sgw)[8], float (&sgb)[8]) {
  float w[8], b[8], s[8], g[8];
  vector8<T, WHOLE>(unmoved(a.w1), column(v), a.dim, 1.0f, w);
  vector8<T, WHOLE>(unmoved(a.b1), column(v), a.dim, 0.0f, b);
  vector8<T, WHOLE>(unmoved(a.scale), column(v), a.dim, 1.0f, s);
  vector8<T, WHOLE>(unmoved(gate), column(v), a.dim, 1.0f, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    sgw[j] = s[j] * g[j] * w[j];
    sgb[j] = s[j] * g[j] * b[j];
  }
}
template <typename T, bool WHOLE, int NV>
__device__ __forceinline__ void products(const JoinArgs &a, const T *gate, Row<NV> &sgw, Row<NV> &sgb) {
#pragma unroll
  for (int v = 0; v < NV; ++v) product8<T, WHOLE>(a, gate, v, sgw.v[v], sgb.v[v]);
}

// A block takes a run of rows, each thread NV pieces of 8 columns of a row; the
// next row's loads are issued before the current row's sums, and the vectors'
// products are formed once per gate row. WHOLE: rows of whole pieces; the code for
// a row's end, which is there for every tensor, costs 16384 x 1280 bf16 4 of 49 us
// (backward 25 of 91) even where no row has one. In a training pass that shape takes 44
// us, 168 MB at 3.8 TB/s with the waves waiting 67 % of their time: bound by HBM and by a
// row's chain of sums. Called again and again on the same inputs, which the memory-side
// cache then holds, it takes 32 us. The generator, 20 32 x 32 products and 40 other
// instructions per 8 elements, is 3.5 us of either.
template <typename T, int NV, bool BIAS, bool WHOLE>
__global__ __launch_bounds__(512) void k_join_fwd(JoinArgs a) {
  __shared__ RowSums sh;
  row_sums_init(sh);
  int turn = 0;
  const Rng rng = a.drop16 ? load_rng(a.rng, a.site) : Rng{};
  const int64_t r0 = blockIdx.x * a.per_block, r1 = min(a.rows, r0 + a.per_block);
  Raw<T> nx[NV], nf[NV];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      nx[v] = piece_of<WHOLE>(static_cast<const T *>(a.x) + row * a.ldx, column(v), a.dim);
      if (a.f) nf[v] = piece_of<WHOLE>(static_cast<const T *>(a.f) + row * a.ldf, column(v), a.dim);
    }
  };
  if (r0 < r1) fetch(r0);
  Row<NV> sgw, sgb, w2, b2;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    vector8<T, WHOLE>(a.w2, column(v), a.dim, 1.0f, w2.v[v]);
    if constexpr (BIAS) vector8<T, WHOLE>(a.b2, column(v), a.dim, 0.0f, b2.v[v]);
  }
  int64_t gate_row = a.gate ? r0 / a.gate_run : 0, gate_end = a.gate ? (gate_row + 1) * a.gate_run : a.rows;
  if (a.f && r0 < r1)
    products<T, WHOLE>(a, a.gate ? static_cast<const T *>(a.gate) + gate_row * a.ldg : nullptr, sgw, sgb);
#pragma unroll 1
  for (int64_t row = r0; row < r1; ++row) {
    if (a.f && row == gate_end) {
      ++gate_row;
      gate_end += a.gate_run;
      products<T, WHOLE>(a, static_cast<const T *>(a.gate) + gate_row * a.ldg, sgw, sgb);
    }
    Row<NV> y, u;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      widen<T>(nx[v], y.v[v]);
      if (a.f) widen<T>(nf[v], u.v[v]);
    }
    if (row + 1 < r1) fetch(row + 1);
    if (a.f) {
      const float r = a.post ? norm_of<NV>(u, a, sh, turn) : 1.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float m[8];
        factors<NV == 1>(a, rng, row, column(v), a.k, m);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float t = r * u.v[v][j];
          y.v[v][j] = fmaf(m[j], BIAS ? fmaf(t, sgw.v[v][j], sgb.v[v][j]) : t * sgw.v[v][j], y.v[v][j]);
        }
      }
    }
    if (a.y) {
#pragma unroll
      for (int v = 0; v < NV; ++v) put_piece<WHOLE>(static_cast<T *>(a.y) + row * a.dim, column(v), a.dim, y.v[v]);
    }
    if (a.pre) {
      // (columns past dim hold zeros: the vectors and rows end there)
      const float r = norm_of<NV>(y, a, sh, turn);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float t = r * y.v[v][j];
          y.v[v][j] = BIAS ? fmaf(t, w2.v[v][j], b2.v[v][j]) : t * w2.v[v][j];
        }
        put_piece<WHOLE>(static_cast<T *>(a.z) + row * a.dim, column(v), a.dim, y.v[v]);
      }
    }
  }
}

// Gate rows against a block's rows: one gate row (or none) for all of them, a
// gate row for each, or several gate rows of several rows each (kGroups; kRuns with
// two pieces per thread).
enum GateMode { kOneGate = 0, kEachRow = 1, kGroups = 2, kRuns = 3 };

// A block takes consecutive rows: whole groups (the rows of one gate row), or a
// part of one group where there are fewer groups than blocks. Column sums stay
// in registers over the block's rows and go to the block's partial row.
//
// The vectors leave the sums over rows: with M = D (kOneGate) or D g, P = sum dY
// M f^ and Q = sum dY M, the sums of scale, post_weight and post_bias are k times
// g (w1 P + b1 Q), s g P and s g Q (kOneGate's g; else 1), and one gate row's is
// k s (w1 P + b1 Q). So a row adds to P, and Q where there are biases (BIAS), and
// to dz y^ and dz; several gate rows add a sum of their own (kGroups). Two pieces per
// thread leave no registers for that one: kRuns takes P and Q as of one gate row, and at
// the end of its rows adds what they give to the block's partial rows in memory.
//
// A row has three block sums one after the other (RMS; LAYER five): the next
// row is loaded before them, and the y norm's two sums share one.
//
// 16384 x 1280 in bf16 with both norms, gate, scale and dropout: 68 us, 252 MB of
// tensors and 39 MB of partial rows at 4.2 TB/s; VALU busy half of the time, waves
// waiting 63 % of theirs: bound by a row's chain of sums as much as by HBM.
template <typename T, int NV, int MODE, bool BIAS, bool WHOLE>
__global__ __launch_bounds__(512, NV == 1 && MODE == kOneGate && !BIAS && sizeof(T) == 2 ? 4 : 2)
void k_join_bwd(JoinArgs a) {
  __shared__ RowSums sh;
  row_sums_init(sh);
  int turn = 0;
  const Rng rng = a.drop16 ? load_rng(a.rng, a.site) : Rng{};
  // two pieces per thread: the biases' sums (beside a gate per row all sums) in LDS,
  // each thread its own slots; the registers hold no more
  constexpr bool kLds = NV > 1 && BIAS, kLdsP = kLds && MODE != kOneGate;
  constexpr bool kOne = MODE == kOneGate || MODE == kRuns;       // a gate row for many rows
  constexpr int kSlots = kLdsP ? 4 : kLds ? 2 : 0;
  Row<NV> P = {}, Q = {}, sw2 = {}, sb2 = {}, sg = {};
  __shared__ float4v sums[kLds ? kSlots * 2 * NV * 512 : 1];
  auto slot = [&](int which, int v, int half) -> float4v & {
    return sums[((which * NV + v) * 2 + half) * 512 + threadIdx.x];
  };
  if constexpr (kLds) {
#pragma unroll
    for (int i = 0; i < kSlots * 2 * NV; ++i) slot(i / (2 * NV), (i >> 1) % NV, i & 1) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  }
  auto add = [&](int which, int v, const float (&x)[8], float (&acc)[8]) {
    if constexpr (kLds) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4v t = slot(which, v, h);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] += x[4 * h + j];
        slot(which, v, h) = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += x[j];
    }
  };
  auto take = [&](int which, int v, float (&acc)[8]) {
    if constexpr (kLds) {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = slot(which, v, j >> 2)[j & 3];
    }
  };

  const int64_t blk = blockIdx.x;
  const int64_t g0 = a.parts > 1 ? blk / a.parts : blk * a.gpb;
  const int64_t g1 = a.parts > 1 ? g0 + 1 : min(a.groups, g0 + a.gpb);
  const int64_t r0 = g0 * a.rpg + (a.parts > 1 ? (blk - g0 * a.parts) * a.rpp : 0);
  const int64_t r1 = a.parts > 1 ? min(r0 + a.rpp, g1 * a.rpg) : g1 * a.rpg;
  int64_t gate_row = MODE == kEachRow ? r0 : MODE == kGroups || MODE == kRuns ? g0 : a.gate && r0 < r1 ? r0 / a.gate_run : 0;
  int64_t group_end = MODE == kGroups || MODE == kRuns ? (g0 + 1) * a.rpg : 0;
  const T *gate0 = kOne && a.gate ? static_cast<const T *>(a.gate) + gate_row * a.ldg : nullptr;
  // what P and Q give: a part of the gate row's sum (kRuns: the sum), and parts of those of
  // scale, post_weight and post_bias. fresh: the first ones of the block
  const int64_t step = int64_t(gridDim.x) * a.ldp;
  auto leave = [&](int v, bool fresh) {
    float w[8], b[8], s[8], g[8], t[3][8], dg[8];
    take(0, v, Q.v[v]);
    if constexpr (kLdsP) take(2, v, P.v[v]);
    vector8<T, WHOLE>(unmoved(a.w1), column(v), a.dim, 1.0f, w);
    vector8<T, WHOLE>(unmoved(a.b1), column(v), a.dim, 0.0f, b);
    vector8<T, WHOLE>(unmoved(a.scale), column(v), a.dim, 1.0f, s);
    vector8<T, WHOLE>(unmoved(gate0), column(v), a.dim, 1.0f, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = a.k * (BIAS ? fmaf(w[j], P.v[v][j], b[j] * Q.v[v][j]) : w[j] * P.v[v][j]);
      t[0][j] = a.k * s[j] * g[j] * P.v[v][j];
      t[1][j] = a.k * s[j] * g[j] * Q.v[v][j];
      t[2][j] = g[j] * q;
      dg[j] = s[j] * q;
    }
    if (kOne && a.gpart) put(a.gpart + blk * a.ldp, column(v), a.ldp, dg);
    if (MODE == kRuns && a.dgate) put_piece<WHOLE>(static_cast<T *>(a.dgate) + gate_row * a.dim, column(v), a.dim, dg);
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      float *p = a.part + blk * a.ldp + i * step;
      if (MODE == kRuns && !fresh) {
        float o[8];
        widen<float>(get(p, column(v), a.ldp), o);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[i][j] += o[j];
      }
      put(p, column(v), a.ldp, t[i]);
    }
  };
  Raw<T> nx[NV], nf[NV], nd[NV], nz[NV], ng[NV];
  // two pieces per thread: no loads ahead, each operand not before it is needed,
  // the vectors' products and the dropout factors formed at each use
  constexpr bool kAhead = NV == 1;
  auto fetch_dy = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (a.dy) nd[v] = piece_of<WHOLE>(static_cast<const T *>(a.dy) + row * a.dim, column(v), a.dim);
  };
  auto fetch_gate = [&](int64_t gr) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if constexpr (!kOne) ng[v] = piece_of<WHOLE>(static_cast<const T *>(a.gate) + gr * a.ldg, column(v), a.dim);
  };
  auto fetch = [&](int64_t row, int64_t gr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      nx[v] = piece_of<WHOLE>(static_cast<const T *>(a.x) + row * a.ldx, column(v), a.dim);
      if (a.f) nf[v] = piece_of<WHOLE>(static_cast<const T *>(a.f) + row * a.ldf, column(v), a.dim);
      if (a.dz) nz[v] = piece_of<WHOLE>(static_cast<const T *>(a.dz) + row * a.dim, column(v), a.dim);
      if constexpr (!kAhead && !kOne)
        ng[v] = piece_of<WHOLE>(static_cast<const T *>(a.gate) + gr * a.ldg, column(v), a.dim);
    }
    if (kAhead) {
      fetch_dy(row);
      fetch_gate(gr);
    }
  };
  Row<NV> sgw, sgb, w2;
  if (kAhead && r0 < r1) fetch(r0, gate_row);
  if (kAhead && a.f) products<T, WHOLE>(a, gate0, sgw, sgb);
#pragma unroll
  for (int v = 0; v < NV; ++v) vector8<T, WHOLE>(a.w2, column(v), a.dim, 1.0f, w2.v[v]);
  auto piece = [&](int v) {
    if (!kAhead) {
      __builtin_amdgcn_sched_barrier(0);
      product8<T, WHOLE>(a, gate0, v, sgw.v[v], sgb.v[v]);
    }
  };

#pragma unroll 1
  for (int64_t row = r0; row < r1; ++row) {
    // the next row's gate row
    const bool turns = MODE == kEachRow || (MODE == kGroups && row + 1 == group_end);
    if constexpr (MODE == kRuns) {
      if (row == group_end) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          leave(v, group_end == r0 + a.rpg);
#pragma unroll
          for (int j = 0; j < 8; ++j) P.v[v][j] = Q.v[v][j] = 0.0f;
          if constexpr (kLds) slot(0, v, 0) = slot(0, v, 1) = slot(2, v, 0) = slot(2, v, 1) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        }
        ++gate_row;
        gate0 += a.ldg;
        group_end += a.rpg;
      }
    }
    const int64_t this_gate = gate_row;
    if (turns) ++gate_row;
    if (MODE == kGroups && turns) group_end += a.rpg;
    if (!kAhead) fetch(row, this_gate);
    Row<NV> y, u, d, e, m, g;
    float rf = 1.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      widen<T>(nx[v], y.v[v]);
      if (a.f) widen<T>(nf[v], u.v[v]);
      if (a.dz) widen<T>(nz[v], e.v[v]);
      if constexpr (!kOne) widen<T>(ng[v], g.v[v]);
    }
    auto take_dy = [&]() {
      if (!kAhead) {
        __builtin_amdgcn_sched_barrier(0);
        fetch_dy(row);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (a.dy) {
          widen<T>(nd[v], d.v[v]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) d.v[v][j] = 0.0f;
        }
      }
    };
    if (kAhead) {
      take_dy();
      if (row + 1 < r1) fetch(row + 1, gate_row);
    }
    if (a.f) {
      if (a.post) {
        rf = norm_of<NV>(u, a, sh, turn);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) u.v[v][j] *= rf;
      }
      if (kAhead) {
#pragma unroll
        for (int v = 0; v < NV; ++v) factors<NV == 1>(a, rng, row, column(v), 1.0f, m.v[v]);
      }
    }
    if (a.dz) {
      // y once more, then its norm's gradient; columns past dim hold zeros
      if (a.f) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          piece(v);
          if (!kAhead) factors<NV == 1>(a, rng, row, column(v), 1.0f, m.v[v]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float km = kOne ? a.k * m.v[v][j] : a.k * m.v[v][j] * g.v[v][j];
            y.v[v][j] = fmaf(km, BIAS ? fmaf(u.v[v][j], sgw.v[v][j], sgb.v[v][j]) : u.v[v][j] * sgw.v[v][j], y.v[v][j]);
          }
        }
      }
      if (!kAhead) __builtin_amdgcn_sched_barrier(0);
      float p[2] = {0.0f, 0.0f}, mean = 0.0f;
      if (a.layer) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            p[0] += y.v[v][j];
            p[1] = fmaf(e.v[v][j], w2.v[v][j], p[1]);
          }
        }
        row_sum<2>(p, sh, turn);
        subtract_mean(y, p[0] * a.inv, a.dim);
        mean = p[1] * a.inv;
        p[0] = p[1] = 0.0f;
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          p[0] = fmaf(y.v[v][j], y.v[v][j], p[0]);
          p[1] = fmaf(e.v[v][j] * w2.v[v][j], y.v[v][j], p[1]);
        }
      }
      row_sum<2>(p, sh, turn);
      const float r = __builtin_amdgcn_rsqf(fmaf(p[0], a.inv, a.eps)), mt = p[1] * a.inv * r;
      if (!kAhead) take_dy();
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float ey[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float t = r * y.v[v][j];
          d.v[v][j] = fmaf(r, fmaf(-t, mt, fmaf(e.v[v][j], w2.v[v][j], -mean)), d.v[v][j]);
          if constexpr (kLdsP) ey[j] = e.v[v][j] * t;
          else sw2.v[v][j] = fmaf(e.v[v][j], t, sw2.v[v][j]);
        }
        if constexpr (kLdsP) add(3, v, ey, sw2.v[v]);
        if constexpr (BIAS) add(1, v, e.v[v], sb2.v[v]);
      }
      if (a.layer) {
        // the mean went out of columns past dim as well, and the post norm sums d over a
        // row: zeros there again (masked here, not above: no register more is held)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) d.v[v][j] = column(v) + (WHOLE ? 0 : j) < a.dim ? d.v[v][j] : 0.0f;
      }
    }
    if (!kAhead && !a.dz) take_dy();
    if (a.dx) {
#pragma unroll
      for (int v = 0; v < NV; ++v) put_piece<WHOLE>(static_cast<T *>(a.dx) + row * a.dim, column(v), a.dim, d.v[v]);
    }
    if (!a.f) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float dg[8], du[8];
      piece(v);
      if (!kAhead) factors<NV == 1>(a, rng, row, column(v), 1.0f, m.v[v]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d.v[v][j] *= m.v[v][j];                                  // dY D
        if constexpr (!kOne) {
          const float t = a.k * d.v[v][j];
          dg[j] = t * (BIAS ? fmaf(u.v[v][j], sgw.v[v][j], sgb.v[v][j]) : u.v[v][j] * sgw.v[v][j]);
          if constexpr (MODE == kGroups) dg[j] = sg.v[v][j] += dg[j];
          d.v[v][j] *= g.v[v][j];
        }
        if constexpr (kLdsP) du[j] = d.v[v][j] * u.v[v][j];
        else P.v[v][j] = fmaf(d.v[v][j], u.v[v][j], P.v[v][j]);
      }
      if constexpr (BIAS) add(0, v, d.v[v], Q.v[v]);
      if constexpr (kLdsP) add(2, v, du, P.v[v]);
      // du w1 = k dY M s g w1
#pragma unroll
      for (int j = 0; j < 8; ++j) d.v[v][j] *= a.k * sgw.v[v][j];
      if constexpr (!kOne) {
        if (turns) {
          if (a.dgate) put_piece<WHOLE>(static_cast<T *>(a.dgate) + this_gate * a.dim, column(v), a.dim, dg);
          if constexpr (MODE == kGroups) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sg.v[v][j] = 0.0f;
          }
        }
      }
    }
    if (a.df) {
      if (a.post) {
        float p[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            p[0] = fmaf(d.v[v][j], u.v[v][j], p[0]);
            p[1] += d.v[v][j];
          }
        row_sum<2>(p, sh, turn);
        const float mt = p[0] * a.inv, mean = a.layer ? p[1] * a.inv : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) d.v[v][j] = rf * fmaf(-u.v[v][j], mt, d.v[v][j] - mean);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) put_piece<WHOLE>(static_cast<T *>(a.df) + row * a.dim, column(v), a.dim, d.v[v]);
    }
  }

  if (MODE != kRuns && !a.part && !a.gpart) return;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    leave(v, MODE != kRuns || group_end == r0 + a.rpg);
    if (!a.part) continue;
    take(1, v, sb2.v[v]);
    if constexpr (kLdsP) take(3, v, sw2.v[v]);
    put(a.part + blk * a.ldp + 3 * step, column(v), a.ldp, sw2.v[v]);
    put(a.part + blk * a.ldp + 4 * step, column(v), a.ldp, sb2.v[v]);
  }
}

// Column sums of partial rows: item i (blockIdx.y) below `kinds` is one of the
// vectors, over all blocks; the others are gate rows, over their parts. Latency: 26 MB
// in 7.6 us with 16-byte loads, four ahead (9.5 us with 4-byte ones).
struct SumArgs {
  const float *part, *gpart;
  void *out[5];
  int32_t from[5];                              // which of the five partials
  void *dgate;
  int64_t blocks, parts;
  int32_t kinds, dim, ldp;
};
template <typename T>
__global__ __launch_bounds__(1024) void k_join_sum(SumArgs a) {
  __shared__ __attribute__((aligned(16))) float sh[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const int item = blockIdx.y;
  const float *p;
  int64_t n;
  T *out;
  if (item < a.kinds) {
    p = a.part + a.from[item] * a.blocks * a.ldp;
    n = a.blocks;
    out = static_cast<T *>(a.out[item]);
  } else {
    const int64_t g = item - a.kinds;
    p = a.gpart + g * a.parts * a.ldp;
    n = a.parts;
    out = static_cast<T *>(a.dgate) + g * a.dim;
  }
  // a wave takes four rows at once, 16 bytes of 16 lanes each; four such loads ahead
  const int c4 = blockIdx.x * 64 + (lane & 15) * 4;
  float4v s[4] = {};
  if (c4 < a.ldp) {
    int64_t i = wave * 4 + (lane >> 4);
    for (; i + 192 < n; i += 256)
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += *reinterpret_cast<const float4v *>(p + (i + 64 * q) * a.ldp + c4);
    for (; i < n; i += 64) s[0] += *reinterpret_cast<const float4v *>(p + i * a.ldp + c4);
  }
  s[0] = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s[0][j] += __shfl_xor(s[0][j], 16);
    s[0][j] += __shfl_xor(s[0][j], 32);
  }
  if (lane < 16) *reinterpret_cast<float4v *>(&sh[wave][lane * 4]) = s[0];
  __syncthreads();
  if (wave == 0 && c < a.dim) {
    float t = 0.0f;
    for (int w = 0; w < 16; ++w) t += sh[w][lane];
    out[c] = from_f<T>(t);
  }
}

// Eight elements a thread. HBM bounds it: 403 MB in 72 us, 5.6 TB/s (16384 x 6144 in
// bf16); the generator keeps the VALU busy 43 % of that time, beside the loads.
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(int64_t n, uint32_t drop16, const int64_t *rng_p, int64_t site,
                                                 float keep, const T *x, T *y) {
  const Rng rng = load_rng(rng_p, site);
  const int64_t pieces = (n + 7) >> 3;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
    const int left = int(min(int64_t(8), n - i * 8));
    const Raw<T> r = get(x + i * 8, 0, left);
    float v[8], m[8];
    keep8<false>(i * 8, 0, rng, drop16, keep, m);
    widen<T>(r, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = m[j] != 0.0f ? v[j] * keep : 0.0f;
    put(y + i * 8, 0, left, v);
  }
}

// (nothing dropped)
template <typename T>
__global__ __launch_bounds__(256) void k_copy(int64_t n, const T *x, T *y) {
  const int64_t pieces = (n + 7) >> 3;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
    const int left = int(min(int64_t(8), n - i * 8));
    float v[8];
    widen<T>(get(x + i * 8, 0, left), v);
    put(y + i * 8, 0, left, v);
  }
}

float keep_factor(uint32_t drop) { return float(65536.0 / (65536.0 - double(drop))); }

int join_threads(int dim) { return int(cdiv(std::min(dim, 4096), 512)) * 64; }

JoinArgs join_args(const JoinShape &s, const slorr_join_tensors_t &t, const int64_t *rng) {
  JoinArgs a{};
  a.x = t.x;
  a.f = t.f;
  a.w1 = t.post_weight;
  a.b1 = t.post_bias;
  a.gate = t.f ? t.gate : nullptr;
  a.scale = t.scale;
  a.w2 = t.pre_weight;
  a.b2 = t.pre_bias;
  a.rng = rng;
  a.rows = s.rows;
  a.ldx = s.ldx;
  a.ldf = s.ldf;
  a.ldg = s.ld_gate;
  a.gate_rows = s.gate_rows;
  a.gate_run = a.gate && s.rows ? s.rows / s.gate_rows : 1;
  a.site = s.site;
  a.dim = s.dim;
  a.ldp = int32_t(up8(s.dim));
  a.layer = s.layer;
  a.post = s.post;
  a.pre = s.pre;
  a.drop16 = s.drop << 16;
  a.eps = s.eps;
  a.inv = 1.0f / float(s.dim);
  a.k = s.alpha * keep_factor(s.drop);
  return a;
}

template <typename T, int NV, bool BIAS>
void launch_forward_as(const JoinArgs &a, dim3 grid, dim3 block, hipStream_t st) {
  if (a.dim % 8) hipLaunchKernelGGL((k_join_fwd<T, NV, BIAS, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_join_fwd<T, NV, BIAS, true>), grid, block, 0, st, a);
  check(hipGetLastError(), "kernel launch");
}
template <typename T>
void launch_forward(const JoinArgs &a, uint32_t blocks, int threads, hipStream_t st) {
  const dim3 grid(blocks), block(threads);
  const bool bias = a.b1 || a.b2;
  if (a.dim > 4096 && bias) launch_forward_as<T, 2, true>(a, grid, block, st);
  else if (a.dim > 4096) launch_forward_as<T, 2, false>(a, grid, block, st);
  else if (bias) launch_forward_as<T, 1, true>(a, grid, block, st);
  else launch_forward_as<T, 1, false>(a, grid, block, st);
}

template <typename T, int NV, int MODE, bool BIAS>
void launch_backward_in(const JoinArgs &a, dim3 grid, dim3 block, hipStream_t st) {
  if (a.dim % 8) hipLaunchKernelGGL((k_join_bwd<T, NV, MODE, BIAS, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_join_bwd<T, NV, MODE, BIAS, true>), grid, block, 0, st, a);
  check(hipGetLastError(), "kernel launch");
}
template <typename T, int NV, int MODE>
void launch_backward_as(const JoinArgs &a, int64_t blocks, hipStream_t st) {
  const dim3 grid{uint32_t(blocks)}, block(join_threads(a.dim));
  if (a.b1 || a.b2) launch_backward_in<T, NV, MODE, true>(a, grid, block, st);
  else launch_backward_in<T, NV, MODE, false>(a, grid, block, st);
}
template <typename T, int NV>
void launch_backward_of(const JoinArgs &a, int mode, int64_t blocks, hipStream_t st) {
  if (mode == kEachRow) launch_backward_as<T, NV, kEachRow>(a, blocks, st);
  else if (mode == kGroups) launch_backward_as<T, NV, NV == 1 ? kGroups : kRuns>(a, blocks, st);
  else launch_backward_as<T, NV, kOneGate>(a, blocks, st);
}
template <typename T>
void launch_backward(const JoinArgs &a, int mode, int64_t blocks, hipStream_t st) {
  if (a.dim > 4096) launch_backward_of<T, 2>(a, mode, blocks, st);
  else launch_backward_of<T, 1>(a, mode, blocks, st);
}

}  // namespace

JoinCut join_cut(const JoinShape &s) {
  JoinCut c;
  // as many blocks as the CUs hold at once, by the kernels' registers: 16 waves per
  // CU with bf16 rows of one piece per thread, else 8 (us of k_join_bwd and k_join_sum
  // with 4 blocks per CU whatever their size, and so: 65536 x 512 bf16 189, 113; 4096 x
  // 4096 bf16 75, 59; 4096 x 6144 bf16 189, 144; 8192 x 4096 fp32 224, 197; 16384 x 1280
  // bf16 77, 74)
  const int waves = s.dim <= 4096 && s.dtype == SLORR_BF16 ? 16 : 8;
  const int64_t target = int64_t(kCus) * std::max(1, waves * 64 / join_threads(s.dim));
  const bool summed = s.gate_rows > 1 && s.gate_rows < s.rows;     // gate rows of several tokens each
  c.groups = summed ? s.gate_rows : 1;
  c.rows_per_group = s.rows / c.groups;
  if (c.groups >= target) {
    c.groups_per_block = cdiv(c.groups, target);
    c.parts = 1;
    c.rows_per_part = c.rows_per_group;
    c.blocks = cdiv(c.groups, c.groups_per_block);
  } else {
    // (parts of at least 4 rows: each leaves partial rows to write and to add)
    c.parts = std::max<int64_t>(1, std::min(cdiv(target, c.groups), cdiv(c.rows_per_group, 4)));
    c.rows_per_part = std::max<int64_t>(1, cdiv(c.rows_per_group, c.parts));
    c.parts = std::max<int64_t>(1, cdiv(c.rows_per_group, c.rows_per_part));
    c.groups_per_block = 1;
    c.blocks = c.groups * c.parts;
  }
  return c;
}

// Partials: five vectors and the gate's sum, a row per block each.
size_t join_workspace(const JoinShape &s) {
  return std::max<size_t>(256, size_t(join_cut(s).blocks) * 6 * size_t(up8(s.dim)) * sizeof(float));
}

void enqueue_join_forward(const JoinShape &s, const slorr_join_tensors_t &t, const int64_t *rng, void *y, void *z,
                          hipStream_t st) {
  if (!s.rows) return;
  JoinArgs a = join_args(s, t, rng);
  a.y = y;
  a.z = z;
  // as many blocks as the CUs hold at once, each a run of rows: 16 waves per CU, 24
  // where the registers allow it (us with 16 and 24: 65536 x 512 bf16 in a training pass
  // 69.5, 53.6; 16384 x 1280 bf16 41.7, 44.2, and called again on inputs that the
  // memory-side cache holds 37.0, 32.1; 4096 x 2048 bf16 17.0, 16.8. 4096 x 6144 bf16,
  // whose blocks are 8 waves: 60 with 8, 49.5 with 16)
  const int threads = join_threads(s.dim);
  const int waves = s.dim <= 4096 && s.dtype == SLORR_BF16 && !a.b1 && !a.b2 ? 24 : 16;
  a.per_block = std::max<int64_t>(1, cdiv(s.rows, kCus * (waves * 64 / threads)));
  const uint32_t grid = uint32_t(cdiv(s.rows, a.per_block));
  if (s.dtype == SLORR_BF16) launch_forward<bf16_t>(a, grid, threads, st);
  else launch_forward<float>(a, grid, threads, st);
}

void enqueue_join_backward(const JoinShape &s, const slorr_join_tensors_t &t, const int64_t *rng, const void *dy,
                           const void *dz, const slorr_join_grads_t &g, void *ws, hipStream_t st) {
  JoinArgs a = join_args(s, t, rng);
  const JoinCut c = join_cut(s);
  a.dy = dy;
  a.dz = dz;
  a.dx = g.x;
  a.df = g.f;
  a.dgate = g.gate;
  a.groups = c.groups;
  a.rpg = c.rows_per_group;
  a.gpb = c.groups_per_block;
  a.parts = c.parts;
  a.rpp = c.rows_per_part;
  float *w = static_cast<float *>(ws);
  const int64_t n = c.blocks * a.ldp;
  SumArgs q{};
  void *const outs[5] = {g.post_weight, g.post_bias, g.scale, g.pre_weight, g.pre_bias};
  for (int i = 0; i < 5; ++i)
    if (outs[i]) {
      q.out[q.kinds] = outs[i];
      q.from[q.kinds++] = i;
    }
  const bool each = a.gate && a.gate_run == 1 && s.gate_rows == s.rows;
  const int mode = each ? kEachRow : a.gate && c.groups > 1 && c.parts == 1 ? kGroups : kOneGate;
  // kOneGate's blocks leave parts of the gate's sums, to be added afterwards (with no
  // token at all: zeros)
  const bool joined = g.gate && (!s.rows || mode == kOneGate);
  a.part = q.kinds ? w : nullptr;
  a.gpart = joined ? w + 5 * n : nullptr;
  if (s.rows) {
    if (s.dtype == SLORR_BF16) launch_backward<bf16_t>(a, mode, c.blocks, st);
    else launch_backward<float>(a, mode, c.blocks, st);
  }
  const int64_t gates = joined ? (s.rows ? c.groups : s.gate_rows) : 0;
  if (!q.kinds && !gates) return;
  q.part = a.part;
  q.gpart = a.gpart;
  q.dgate = g.gate;
  q.blocks = s.rows ? c.blocks : 0;
  q.parts = s.rows ? c.parts : 0;
  q.dim = s.dim;
  q.ldp = a.ldp;
  const uint32_t gx = uint32_t(cdiv(s.dim, 64));
  // grid.y is limited to 65535: gate rows in several launches
  for (int64_t first = 0; first == 0 || first < gates; first += 32768) {
    SumArgs p = q;
    if (first) p.kinds = 0;
    const int64_t take = std::min<int64_t>(gates - first, 32768);
    if (p.gpart) p.gpart += first * q.parts * q.ldp;
    p.dgate = static_cast<char *>(q.dgate) + (q.dgate ? first * s.dim * (s.dtype == SLORR_BF16 ? 2 : 4) : 0);
    const dim3 grid(gx, uint32_t(p.kinds + std::max<int64_t>(take, 0)));
    if (s.dtype == SLORR_BF16) hipLaunchKernelGGL(k_join_sum<bf16_t>, grid, dim3(1024), 0, st, p);
    else hipLaunchKernelGGL(k_join_sum<float>, grid, dim3(1024), 0, st, p);
    check(hipGetLastError(), "kernel launch");
  }
}

void enqueue_dropout(int64_t n, int32_t dtype, uint32_t drop, const int64_t *rng, int64_t site, const void *x,
                     void *y, hipStream_t st) {
  if (!n || (!drop && x == y)) return;
  const dim3 grid(uint32_t(std::min<int64_t>(cdiv(cdiv(n, 8), 256), 32 * kCus))), block(256);
  if (dtype == SLORR_BF16) {
    const bf16_t *p = static_cast<const bf16_t *>(x);
    bf16_t *q = static_cast<bf16_t *>(y);
    if (drop) hipLaunchKernelGGL(k_dropout<bf16_t>, grid, block, 0, st, n, drop << 16, rng, site, keep_factor(drop), p, q);
    else hipLaunchKernelGGL(k_copy<bf16_t>, grid, block, 0, st, n, p, q);
  } else {
    const float *p = static_cast<const float *>(x);
    float *q = static_cast<float *>(y);
    if (drop) hipLaunchKernelGGL(k_dropout<float>, grid, block, 0, st, n, drop << 16, rng, site, keep_factor(drop), p, q);
    else hipLaunchKernelGGL(k_copy<float>, grid, block, 0, st, n, p, q);
  }
  check(hipGetLastError(), "kernel launch");
}

}  // namespace slorr
