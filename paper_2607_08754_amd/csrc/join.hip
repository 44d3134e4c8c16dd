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
#include "device.hpp"
#include "layout.hpp"

namespace slorr {
namespace {

void check(hipError_t e, const char *what) {
  if (e != hipSuccess) throw HipError(std::string(what) + ": " + hipGetErrorString(e));
}
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ generator

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
    c[0] = uint32_t(b >> 32) ^ c[1] ^ k0;
    c[1] = uint32_t(b);
    c[2] = uint32_t(a >> 32) ^ c[3] ^ k1;
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

// Bit j: element e + j is kept. Eight elements from a multiple of 8 on take one
// generator block, others two.
__device__ __forceinline__ uint32_t keep8(int64_t e, const Rng &r, uint32_t drop) {
  uint32_t bits = 0, c[4];
  philox(uint64_t(e) >> 3, r.offset, r.key, c);
#pragma unroll
  for (int j = 0; j < 8; ++j) bits |= uint32_t(((c[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= drop) << j;
  const int s = int(e & 7);
  if (s) {
    uint32_t next = 0;
    philox((uint64_t(e) >> 3) + 1, r.offset, r.key, c);
#pragma unroll
    for (int j = 0; j < 8; ++j) next |= uint32_t(((c[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= drop) << j;
    bits = (bits | next << 8) >> s;
  }
  return bits;
}

// ------------------------------------------------------------------- accesses

// 8 values from column c of a row (zeros past dim). whole: rows are 16-byte
// aligned and dim is a multiple of 8.
template <typename T>
__device__ __forceinline__ void get(const T *row, int c, int dim, bool whole, float (&v)[8]) {
  if (whole) {
    if (c < dim) {
      if constexpr (sizeof(T) == 2) {
        const u32x4 q = gload16(row + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? q[j >> 1] & 0xffff0000u : q[j >> 1] << 16);
      } else {
        const u32x4 a = gload16(row + c), b = gload16(row + c + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j < 4 ? a[j & 3] : b[j & 3]);
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = c + j < dim ? to_f(row[c + j]) : 0.0f;
}

template <typename T>
__device__ __forceinline__ void put(T *row, int c, int dim, bool whole, const float (&v)[8]) {
  if (whole) {
    if (c >= dim) return;
    if constexpr (sizeof(T) == 2) {
      typedef float floatx8 __attribute__((ext_vector_type(8)));
      typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
      floatx8 f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = v[j];
      gstore16(row + c, __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8)));
    } else {
      u32x4 a, b;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = __float_as_uint(v[j]);
        b[j] = __float_as_uint(v[4 + j]);
      }
      gstore16(row + c, a);
      gstore16(row + c + 4, b);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (c + j < dim) row[c + j] = from_f<T>(v[j]);
}

// Sums of K values over the block, the result in every thread: butterfly within
// each wave, then the waves' sums in wave order. sh: two buffers, used in turn
// (a wave that writes one again has passed the barrier after the other's reads).
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float (*sh)[8][K], int &turn) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o);
  const int waves = int(blockDim.x) >> 6;
  if (waves == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) sh[turn][threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0f;
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += sh[turn][w][k];
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
  int64_t groups, rpg, gpb, parts, rpp;         // JoinCut
  int64_t site;
  int32_t dim, ldp, layer, post, pre;
  uint32_t drop;
  float eps, alpha, keep;                       // keep: 1 / (1 - p')
  int32_t wx, wf, wg, wd;                       // whole (see get): x, f, gate, contiguous tensors
};

// The normalised row in place; returns r.
template <int NV>
__device__ __forceinline__ float normalise(float (&t)[NV][8], const JoinArgs &a, float (*sh)[8][2], int &turn) {
  const float inv = 1.0f / float(a.dim);
  float q[2] = {0.0f, 0.0f};
  if (a.layer) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) q[0] += t[v][j];
    row_sum<2>(q, sh, turn);
    const float mu = q[0] * inv;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) t[v][j] = c + j < a.dim ? t[v][j] - mu : 0.0f;
    }
    q[0] = q[1] = 0.0f;
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) q[0] = fmaf(t[v][j], t[v][j], q[0]);
  row_sum<2>(q, sh, turn);
  const float r = 1.0f / sqrtf(fmaf(q[0], inv, a.eps));
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) t[v][j] *= r;
  return r;
}

// A norm's input gradient r (A - mean A - t^ mean(A t^)) in place of A.
template <int NV>
__device__ __forceinline__ void norm_back(float (&A)[NV][8], const float (&t)[NV][8], float r, const JoinArgs &a,
                                          float (*sh)[8][2], int &turn) {
  const float inv = 1.0f / float(a.dim);
  float q[2] = {0.0f, 0.0f};
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      q[0] = fmaf(A[v][j], t[v][j], q[0]);
      q[1] += A[v][j];
    }
  row_sum<2>(q, sh, turn);
  const float mt = q[0] * inv, m = a.layer ? q[1] * inv : 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) A[v][j] = r * (A[v][j] - m - t[v][j] * mt);
}

template <typename T>
__device__ __forceinline__ void vec(const void *p, int c, const JoinArgs &a, float none, float (&v)[8]) {
  if (p) {
    get(static_cast<const T *>(p), c, a.dim, a.wd, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = none;
  }
}

// alpha D of 8 elements of a row
__device__ __forceinline__ void factors(const JoinArgs &a, const Rng &rng, int64_t row, int c, float (&m)[8]) {
  uint32_t bits = 0xffu;
  if (a.drop) bits = keep8(row * a.dim + c, rng, a.drop);
  const float k = a.drop ? a.alpha * a.keep : a.alpha;
#pragma unroll
  for (int j = 0; j < 8; ++j) m[j] = (bits >> j) & 1u ? k : 0.0f;
}

template <typename T, int NV>
__global__ __launch_bounds__(512) void k_join_fwd(JoinArgs a) {
  __shared__ float sh[2][8][2];
  int turn = 0;
  const Rng rng = a.drop ? load_rng(a.rng, a.site) : Rng{};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float y[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
      get(static_cast<const T *>(a.x) + row * a.ldx, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a.dim, a.wx, y[v]);
    if (a.f) {
      float u[NV][8];
#pragma unroll
      for (int v = 0; v < NV; ++v)
        get(static_cast<const T *>(a.f) + row * a.ldf, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a.dim, a.wf, u[v]);
      if (a.post) normalise<NV>(u, a, sh, turn);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
        float w[8], b[8], s[8], g[8], m[8];
        vec<T>(a.w1, c, a, 1.0f, w);
        vec<T>(a.b1, c, a, 0.0f, b);
        vec<T>(a.scale, c, a, 1.0f, s);
        if (a.gate) get(static_cast<const T *>(a.gate) + row / a.gate_run * a.ldg, c, a.dim, a.wg, g);
        factors(a, rng, row, c, m);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          y[v][j] = fmaf(m[j] * s[j] * (a.gate ? g[j] : 1.0f), fmaf(u[v][j], w[j], b[j]), y[v][j]);
      }
    }
    if (a.y) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        put(static_cast<T *>(a.y) + row * a.dim, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a.dim, a.wd, y[v]);
    }
    if (a.pre) {
      // columns past dim hold zeros, but for a bias's sake: keep them out of the sums
      normalise<NV>(y, a, sh, turn);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
        float w[8], b[8];
        vec<T>(a.w2, c, a, 1.0f, w);
        vec<T>(a.b2, c, a, 0.0f, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] = fmaf(y[v][j], w[j], b[j]);
        put(static_cast<T *>(a.z) + row * a.dim, c, a.dim, a.wd, y[v]);
      }
    }
  }
}

// A block takes consecutive rows: whole groups (the rows of one gate row), or a
// part of one group where there are fewer groups than blocks. Column sums stay
// in registers over the block's rows and go to the block's partial row; the
// gate's sum is flushed at each group's end.
template <typename T, int NV>
__global__ __launch_bounds__(512) void k_join_bwd(JoinArgs a) {
  __shared__ float sh[2][8][2];
  int turn = 0;
  const Rng rng = a.drop ? load_rng(a.rng, a.site) : Rng{};
  float sw1[NV][8] = {}, ss[NV][8] = {}, sg[NV][8] = {}, sw2[NV][8] = {};
  // the biases' sums: with two pieces per thread in LDS, where the registers
  // hold no more (each thread its own 16-byte slots)
  constexpr bool kLds = NV > 1;
  float sb1[NV][8] = {}, sb2[NV][8] = {};
  __shared__ float4v bias_acc[kLds ? 4 * NV * 512 : 1];
  auto bias_slot = [&](int which, int v, int half) -> float4v & {
    return bias_acc[((which * NV + v) * 2 + half) * 512 + threadIdx.x];
  };
  if constexpr (kLds) {
#pragma unroll
    for (int i = 0; i < 2 * NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) bias_slot(i / NV, i % NV, h) = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  }
  auto bias_add = [&](int which, int v, const float (&x)[8], float (&acc)[8]) {
    if constexpr (kLds) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4v t = bias_slot(which, v, h);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] += x[4 * h + j];
        bias_slot(which, v, h) = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += x[j];
    }
  };
  auto bias_get = [&](int which, int v, float (&acc)[8]) {
    if constexpr (kLds) {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = bias_slot(which, v, j >> 2)[j & 3];
    }
  };
  const bool each = a.gate && a.gate_run == 1;             // a gate row per row: no sum
  const int64_t blk = blockIdx.x;
  const int64_t g0 = a.parts > 1 ? blk / a.parts : blk * a.gpb;
  const int64_t g1 = a.parts > 1 ? g0 + 1 : min(a.groups, g0 + a.gpb);
  for (int64_t grp = g0; grp < g1; ++grp) {
    const int64_t r0 = grp * a.rpg + (a.parts > 1 ? (blk - g0 * a.parts) * a.rpp : 0);
    const int64_t r1 = a.parts > 1 ? min(r0 + a.rpp, (grp + 1) * a.rpg) : r0 + a.rpg;
    for (int64_t row = r0; row < r1; ++row) {
      float y[NV][8], u[NV][8], d[NV][8];                  // y, then y^; f, then f^; dY
      float r1f = 1.0f, r2 = 1.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
        get(static_cast<const T *>(a.x) + row * a.ldx, c, a.dim, a.wx, y[v]);
        if (a.f) get(static_cast<const T *>(a.f) + row * a.ldf, c, a.dim, a.wf, u[v]);
        if (a.dy) get(static_cast<const T *>(a.dy) + row * a.dim, c, a.dim, a.wd, d[v]);
        else
#pragma unroll
          for (int j = 0; j < 8; ++j) d[v][j] = 0.0f;
      }
      if (a.f && a.post) r1f = normalise<NV>(u, a, sh, turn);
      if (a.pre && a.dz) {
        float A[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
          get(static_cast<const T *>(a.dz) + row * a.dim, c, a.dim, a.wd, A[v]);
          if (a.f) {
            float w[8], b[8], s[8], g[8], m[8];
            vec<T>(a.w1, c, a, 1.0f, w);
            vec<T>(a.b1, c, a, 0.0f, b);
            vec<T>(a.scale, c, a, 1.0f, s);
            if (a.gate) get(static_cast<const T *>(a.gate) + row / a.gate_run * a.ldg, c, a.dim, a.wg, g);
            factors(a, rng, row, c, m);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              y[v][j] = fmaf(m[j] * s[j] * (a.gate ? g[j] : 1.0f), fmaf(u[v][j], w[j], b[j]), y[v][j]);
          }
        }
        r2 = normalise<NV>(y, a, sh, turn);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          float w[8];
          vec<T>(a.w2, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a, 1.0f, w);
          bias_add(1, v, A[v], sb2[v]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sw2[v][j] = fmaf(A[v][j], y[v][j], sw2[v][j]);
            A[v][j] *= w[j];
          }
        }
        norm_back<NV>(A, y, r2, a, sh, turn);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) d[v][j] += A[v][j];
      }
      if (a.dx) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
          put(static_cast<T *>(a.dx) + row * a.dim, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a.dim, a.wd, d[v]);
      }
      if (!a.f) continue;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
        float w[8], b[8], s[8], g[8], m[8], dg[8], du[8];
        vec<T>(a.w1, c, a, 1.0f, w);
        vec<T>(a.b1, c, a, 0.0f, b);
        vec<T>(a.scale, c, a, 1.0f, s);
        if (a.gate) get(static_cast<const T *>(a.gate) + row / a.gate_run * a.ldg, c, a.dim, a.wg, g);
        factors(a, rng, row, c, m);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float gj = a.gate ? g[j] : 1.0f, dm = d[v][j] * m[j];
          const float t = dm * fmaf(u[v][j], w[j], b[j]);
          ss[v][j] = fmaf(t, gj, ss[v][j]);
          dg[j] = t * s[j];
          sg[v][j] += dg[j];
          du[j] = dm * s[j] * gj;
          sw1[v][j] = fmaf(du[j], u[v][j], sw1[v][j]);
          d[v][j] = du[j] * w[j];
        }
        bias_add(0, v, du, sb1[v]);
        if (each && a.dgate) put(static_cast<T *>(a.dgate) + row * a.dim, c, a.dim, a.wd, dg);
      }
      if (a.df) {
        if (a.post) norm_back<NV>(d, u, r1f, a, sh, turn);
#pragma unroll
        for (int v = 0; v < NV; ++v)
          put(static_cast<T *>(a.df) + row * a.dim, (v * int(blockDim.x) + int(threadIdx.x)) * 8, a.dim, a.wd, d[v]);
      }
    }
    if (a.dgate && !each) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
        if (a.gpart) put(a.gpart + blk * a.ldp, c, a.ldp, true, sg[v]);
        else put(static_cast<T *>(a.dgate) + grp * a.dim, c, a.dim, a.wd, sg[v]);
#pragma unroll
        for (int j = 0; j < 8; ++j) sg[v][j] = 0.0f;
      }
    }
  }
  if (a.part) {
    const int64_t step = int64_t(gridDim.x) * a.ldp;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * int(blockDim.x) + int(threadIdx.x)) * 8;
      float *p = a.part + blk * a.ldp;
      bias_get(0, v, sb1[v]);
      bias_get(1, v, sb2[v]);
      put(p, c, a.ldp, true, sw1[v]);
      put(p + step, c, a.ldp, true, sb1[v]);
      put(p + 2 * step, c, a.ldp, true, ss[v]);
      put(p + 3 * step, c, a.ldp, true, sw2[v]);
      put(p + 4 * step, c, a.ldp, true, sb2[v]);
    }
  }
}

// Column sums of partial rows: item i (blockIdx.y) below `kinds` is one of the
// vectors, over all blocks; the others are gate rows, over their parts.
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
  __shared__ float sh[16][64];
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
  float s[4] = {};
  if (c < a.dim) {
    int64_t i = wave;
    for (; i + 48 < n; i += 64)
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += p[(i + 16 * q) * a.ldp + c];
    for (; i < n; i += 16) s[0] += p[i * a.ldp + c];
  }
  sh[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (wave == 0 && c < a.dim) {
    float t = 0.0f;
    for (int w = 0; w < 16; ++w) t += sh[w][lane];
    out[c] = from_f<T>(t);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_dropout(int64_t n, uint32_t drop, const int64_t *rng_p, int64_t site,
                                                 float keep, const T *x, T *y) {
  const Rng rng = load_rng(rng_p, site);
  const int64_t pieces = (n + 7) >> 3;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
    const int left = int(min(int64_t(8), n - i * 8));
    float v[8];
    get(x + i * 8, 0, left, left == 8, v);
    const uint32_t bits = keep8(i * 8, rng, drop);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (bits >> j) & 1u ? v[j] * keep : 0.0f;
    put(y + i * 8, 0, left, left == 8, v);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_copy(int64_t n, const T *x, T *y) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) y[i] = x[i];
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
  a.drop = s.drop;
  a.eps = s.eps;
  a.alpha = s.alpha;
  a.keep = keep_factor(s.drop);
  const int64_t per = s.dtype == SLORR_BF16 ? 8 : 4;       // elements per 16 bytes
  const bool whole = s.dim % 8 == 0;
  a.wd = whole;
  a.wx = whole && s.ldx % per == 0;
  a.wf = whole && s.ldf % per == 0;
  a.wg = whole && s.ld_gate % per == 0;
  return a;
}

}  // namespace

JoinCut join_cut(const JoinShape &s) {
  JoinCut c;
  const int64_t target = 4 * kCus;
  const bool summed = s.gate_rows > 1 && s.gate_rows < s.rows;     // gate rows of several tokens each
  c.groups = summed ? s.gate_rows : 1;
  c.rows_per_group = s.rows / c.groups;
  if (c.groups >= target) {
    c.groups_per_block = cdiv(c.groups, target);
    c.parts = 1;
    c.rows_per_part = c.rows_per_group;
    c.blocks = cdiv(c.groups, c.groups_per_block);
  } else {
    c.parts = std::max<int64_t>(1, std::min(cdiv(target, c.groups), c.rows_per_group));
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
  const dim3 grid(uint32_t(std::min<int64_t>(s.rows, 16 * kCus))), block(join_threads(s.dim));
  const bool two = s.dim > 4096;
  if (s.dtype == SLORR_BF16) {
    if (two) hipLaunchKernelGGL((k_join_fwd<bf16_t, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_join_fwd<bf16_t, 1>), grid, block, 0, st, a);
  } else {
    if (two) hipLaunchKernelGGL((k_join_fwd<float, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_join_fwd<float, 1>), grid, block, 0, st, a);
  }
  check(hipGetLastError(), "kernel launch");
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
  // the gate's sums are joined afterwards where a gate row's tokens are spread
  // over blocks, and where there is no token to write them
  const bool joined = g.gate && (!s.rows || (!each && c.parts > 1));
  a.part = q.kinds ? w : nullptr;
  a.gpart = joined ? w + 5 * n : nullptr;
  if (s.rows) {
    const dim3 grid{uint32_t(c.blocks)}, block(join_threads(s.dim));
    const bool two = s.dim > 4096;
    if (s.dtype == SLORR_BF16) {
      if (two) hipLaunchKernelGGL((k_join_bwd<bf16_t, 2>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_join_bwd<bf16_t, 1>), grid, block, 0, st, a);
    } else {
      if (two) hipLaunchKernelGGL((k_join_bwd<float, 2>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_join_bwd<float, 1>), grid, block, 0, st, a);
    }
    check(hipGetLastError(), "kernel launch");
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
  const int64_t pieces = drop ? cdiv(n, 8) : n;
  const dim3 grid(uint32_t(std::min<int64_t>(cdiv(pieces, 256), 32 * kCus))), block(256);
  if (dtype == SLORR_BF16) {
    const bf16_t *p = static_cast<const bf16_t *>(x);
    bf16_t *q = static_cast<bf16_t *>(y);
    if (drop) hipLaunchKernelGGL(k_dropout<bf16_t>, grid, block, 0, st, n, drop, rng, site, keep_factor(drop), p, q);
    else hipLaunchKernelGGL(k_copy<bf16_t>, grid, block, 0, st, n, p, q);
  } else {
    const float *p = static_cast<const float *>(x);
    float *q = static_cast<float *>(y);
    if (drop) hipLaunchKernelGGL(k_dropout<float>, grid, block, 0, st, n, drop, rng, site, keep_factor(drop), p, q);
    else hipLaunchKernelGGL(k_copy<float>, grid, block, 0, st, n, p, q);
  }
  check(hipGetLastError(), "kernel launch");
}

}  // namespace slorr
