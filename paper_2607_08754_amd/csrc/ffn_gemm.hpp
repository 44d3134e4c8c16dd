// The products of the gated feed-forward block on bf16 MFMA (device code).
//
//   forward   a = x Wg^T, b = x Wu^T, h = act(a) b     one kernel, both products
//             y = h Wd^T
//   backward  dh = dy Wd, then da = dh b act'(a), db = dh act(a) and h again
//             in the same kernel;
//             dx = da Wg + db Wu (one sum over both)
//             dWg = da^T x, dWu = db^T x, dWd = dy^T h (one launch)
//
// Every product is C = A B^T with A, B given either by rows (k contiguous) or
// as [k][row] (transposed while it is read from LDS), so no operand is
// transposed in memory.
//
// fp32 operands are held as three bf16 numbers (planes) hi + mid + lo, which
// carry all 24 significand bits of values from 2^-110 on (bf16's smallest number is
// 2^-133: smaller values are off by half of that); a product is the sum
// of the six plane products whose terms reach 2^-24 of it, the small ones
// first: lo hi, mid mid, hi lo, mid hi, hi mid, hi hi. The kernels run them as six passes
// over k into one accumulator. fp32 MFMA has 1/16 of the bf16 rate: six bf16
// products cost 6/16 of one fp32 product. An infinity gives NaN (infinity times
// a zero plane).
//
// bf16 tensors: h, and da and db in the backward pass, are rounded to bf16 between the
// products, because the matrix instructions take bf16 operands: a second plane would
// double y's, dx's and the weight gradients' products. The roundings are independent
// of the result's own: outputs are off by 2.35e-3 of their size (rms) where one
// rounding of the exact ones is 1.66e-3.
#pragma once
#include "cut.hpp"
#include "device.hpp"

namespace slorr {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));

struct FfnProb {               // one product C (m x n) = sum over sources of A B^T
  const char *a[2], *b[2];     // sources; kAct: b[0], b[1] are both products' rows, one source
  int64_t pa, pb;              // bytes from one plane to the next
  int64_t lda, ldb;            // elements per row
  int32_t m, n, k, nsrc;
  int32_t tm, tn;              // tiles
  int32_t tile0;               // the first tile of this product in the launch
  void *out;
  int64_t ldo;
};

// act(a) and its derivative. fp32 results take the accurate exponential; for bf16
// results the hardware's (errors near 2^-20) is far below the rounding that
// follows.
template <bool F32>
__device__ __forceinline__ float sigmoid(float a) {
  return __builtin_amdgcn_rcpf(1.0f + (F32 ? expf(-a) : __expf(-a)));
}
template <bool F32, int ACT>
__device__ __forceinline__ void act_and_slope(float a, float &f, float &s) {
  if constexpr (ACT == SLORR_SILU) {
    const float g = sigmoid<F32>(a);
    f = a * g;
    s = g * (1.0f + a * (1.0f - g));
  } else if constexpr (ACT == SLORR_GELU) {
    const float c = 0.5f * (1.0f + erff(a * 0.70710678118654752f));
    f = a * c;
    s = c + a * (F32 ? expf(-0.5f * a * a) : __expf(-0.5f * a * a)) * 0.39894228040143268f;
  } else {                     // 0.5 a (1 + tanh u) = a sigmoid(2 u)
    // (a^2 held below infinity: g is 0 or 1 long before, and the slope has 0 times it)
    const float k = 1.5957691216057308f, q = fminf(0.044715f * a * a, 1e30f);
    const float g = sigmoid<F32>(k * a * (1.0f + q));
    f = a * g;
    s = g + f * (1.0f - g) * k * (1.0f + 3.0f * q);
  }
}
// The activation chosen once for a run of values: a choice per value keeps the
// values' chains of dependent instructions from overlapping.
template <typename F>
__device__ __forceinline__ void with_act(int act, F run) {
  if (act == SLORR_SILU) run(std::integral_constant<int, SLORR_SILU>{});
  else if (act == SLORR_GELU) run(std::integral_constant<int, SLORR_GELU>{});
  else run(std::integral_constant<int, SLORR_GELU_TANH>{});
}

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

// 8 values as bf16 (one rounding), or as three planes `plane` bytes apart: each is
// the nearest bf16 number to what the ones before it leave (the first one held
// to the finite range, so that the largest fp32 values leave something finite; an
// infinity or a NaN stays one in the second plane).
template <bool F32>
__device__ __forceinline__ void store_planes(char *p, int64_t plane, const float (&v)[8]) {
  floatx8 f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = v[j];
  if constexpr (!F32) {
    *reinterpret_cast<bf16x8 *>(p) = __builtin_convertvector(f, bf16x8);
  } else {
    constexpr float kMost = 3.38953139e38f;            // the largest bf16 number
    floatx8 c;
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = fminf(fmaxf(f[j], -kMost), kMost);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      const bf16x8 h = __builtin_convertvector(q == 0 ? c : f, bf16x8);
      *reinterpret_cast<bf16x8 *>(p + q * plane) = h;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] -= float(h[j]);
    }
  }
}

// 8 values of the tensors' type, 16-byte aligned and whole.
template <bool F32>
__device__ __forceinline__ void store_whole(void *base, int64_t at, const float (&v)[8]) {
  if constexpr (!F32) {
    store_planes<false>(static_cast<char *>(base) + at * 2, 0, v);
  } else {
    float4v *p = reinterpret_cast<float4v *>(static_cast<float *>(base) + at);
    p[0] = float4v{v[0], v[1], v[2], v[3]};
    p[1] = float4v{v[4], v[5], v[6], v[7]};
  }
}
template <bool F32>
__device__ __forceinline__ void load_whole(const void *base, int64_t at, float (&v)[8]) {
  if constexpr (!F32) {
    const bf16x8 h = *reinterpret_cast<const bf16x8 *>(static_cast<const char *>(base) + at * 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = float(h[j]);
  } else {
    const float4v *p = reinterpret_cast<const float4v *>(static_cast<const float *>(base) + at);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p[j >> 2][j & 3];
  }
}
// a and b as kept for the backward pass. fp32 tensors: as they are. bf16 tensors:
// 16-bit integers with one power of two per 8 values, a step of 2^-15 of the
// largest of the eight at most. bf16 would be as long, but the gradients of a
// and b would carry its rounding twice more (the gradients of a block of 16384
// x 1536 x 6144 are off by 3.5e-3 of their size with it; one rounding of the
// exact ones is 1.7e-3). Eight values with an infinity or a NaN among them are
// kept in bf16, marked by the exponent 255.
// The exponents of a row's 128 columns lie together, those of the next row's same
// columns behind them: what a tile writes and reads of them is contiguous.
struct Kept {
  void *v;                     // a or b: rows of ldf values
  uint8_t *e;
  int64_t rows;
  int32_t ldf;
  __device__ __forceinline__ int64_t at(int row, int col) const { return int64_t(row) * ldf + col; }
  __device__ __forceinline__ int64_t exp_at(int row, int col) const {
    return (int64_t(col >> 7) * rows + row) * 16 + ((col & 127) >> 3);
  }
};
template <bool F32>
__device__ __forceinline__ void store_kept(const Kept &k, int row, int col, const float (&v)[8]) {
  if constexpr (F32) {
    store_whole<true>(k.v, k.at(row, col), v);
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    const int e = max(int(m >> 23), 1);
    u16x8 q;
    if (e == 255) {
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = f32_to_bf16(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = uint16_t(int16_t(min(rintf(ldexpf(v[j], 141 - e)), 32767.0f)));
    }
    // (not read before the backward pass: the caches keep what this launch and the
    // next one read)
    __builtin_nontemporal_store(q, reinterpret_cast<u16x8 *>(static_cast<uint16_t *>(k.v) + k.at(row, col)));
    k.e[k.exp_at(row, col)] = uint8_t(e);
  }
}
// Eight kept values as loaded, for a load issued ahead of its use.
template <bool F32>
struct KeptRaw {
  u32x4 q[F32 ? 2 : 1];
  uint32_t e;
  __device__ __forceinline__ void load(const Kept &k, int row, int col) {
    if constexpr (F32) {
      const float *p = static_cast<const float *>(k.v) + k.at(row, col);
      q[0] = gload16(p);
      q[1] = gload16(p + 4);
    } else {
      q[0] = gload16(static_cast<const uint16_t *>(k.v) + k.at(row, col));
      e = *(const SLORR_GLOBAL uint8_t *)(k.e + k.exp_at(row, col));
    }
  }
  // values 4 i to 4 i + 3 (bf16 tensors)
  __device__ __forceinline__ void half(int i, float4v &v) const {
    if (e == 255) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = to_f(bf16_t(q[0][2 * i + (j >> 1)] >> (16 * (j & 1))));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = ldexpf(float(int16_t(q[0][2 * i + (j >> 1)] >> (16 * (j & 1)))), int(e) - 141);
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(q[j >> 2][j & 3]);
    } else if (e == 255) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = to_f(bf16_t(q[0][j >> 1] >> (16 * (j & 1))));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = ldexpf(float(int16_t(q[0][j >> 1] >> (16 * (j & 1)))), int(e) - 141);
    }
  }
};
// the first n of 8 values (8: whole when the address allows it)
template <bool F32>
__device__ __forceinline__ void store_some(void *base, int64_t at, int n, const float (&v)[8]) {
  using T = typename std::conditional<F32, float, uint16_t>::type;
  T *p = static_cast<T *>(base) + at;
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    store_whole<F32>(base, at, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = from_f<T>(v[j]);
}

// A launch's tiles (those of all its products, with `slabs` slabs of k each): the
// first `whole` are a block's each. The `tail` others are cut along k into `parts`
// parts of `per` slabs, a block's each, the first parts of all of them ahead of
// the second ones: blocks that run together work on the same k and share operand
// panels in L2. (Cut end to end into runs of equal length, whatever their k, the
// weight gradients of 16384 x 1536 x 6144 took 2.66 us a slab instead of 1.73.)
// A part's block stores its fp32 sums, and k_tail adds a tile's parts in order.
struct FfnArgs {
  FfnProb p[3];
  int32_t nprob, act;
  int32_t whole, tail, slabs, parts, per;
  float *part;
  int32_t ldf;                 // row length of the inner tensors
  Kept a, b;                   // as kept for the backward pass (kAct: v may be null)
  char *h, *da, *db;           // bf16 planes
  int64_t plane;               // bytes from one plane of h, da, db to the next
};

// ---------------------------------------------------------------------------
// Block tile BM x BN, wave tiles of FM x FN MFMA tiles of 32 x 32, slabs of 64
// k in NS LDS stages: slab i + NS - 1 is fetched while slab i is multiplied;
// each is waited for by count, then one block barrier publishes it and frees
// the stage of the slab before it.
//
// LDS stages: an operand given by rows is 128-byte rows of 64 k (swz); one
// given as [k][row] is 64 k-rows of 2 BM (2 BN) bytes (kn_off), read with the
// transposing LDS load. Fetches go through buffer resources whose size ends at
// the operand's last valid byte from the slab's corner on: rows past the end
// read as zeros, as do [k][row] k past the end; chunks past the end of a
// row's k are sent outside the resource by their offset.
//
// kAct: each wave's 64 columns are 32 columns of a and the same 32 of b, by
// the order in which the rows of Wg and Wu are placed in the stage.
//
// What bounds it, at 16384 x 1536 x 6144 in bf16: MFMA under the power limit in the
// 256-tiles' loop (1.77 us a slab over all CUs, 1.2 PFLOP/s, MFMA busy 53-57 % at
// 1.8-1.9 GHz: the weights' gradients 859 us, dx 557, y 297); then the ends of tiles
// that move inner tensors, which nothing overlaps (a block's stages leave no LDS for
// a second one): a and b 632 us, where two products as long as dh's take 510; dh 477
// us, of which 38 in each of 6 rounds go for the 1 GB of a, b, h, da and db.
// 128-tiles, of which two share a CU, were no faster at it (12 rounds of 49 us), nor
// when every second block started half a tile later.
template <int BM_, int BN_, int WGM_, int WGN_, int NS_, bool AK, bool BK>
struct FfnTile {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, NS = NS_;
  static constexpr int kWaves = WGM * WGN, kThreads = 64 * kWaves;
  static constexpr int WTM = BM / WGM, WTN = BN / WGN, FM = WTM / 32, FN = WTN / 32;
  static constexpr int kStageA = BM * 128, kStage = kStageA + BN * 128;
  static constexpr int kFW = 4;                        // waves that fetch (one per SIMD)
  static constexpr int kLoadsA = BM / 8 / kFW, kLoadsB = BN / 8 / kFW;
  static constexpr int kPitch = WTN + 4;               // floats per staged row of the epilogue
  static constexpr int kEpi = kWaves * 32 * kPitch * 4;
  static constexpr int kSmem = NS * kStage > kEpi ? NS * kStage : kEpi;
  static_assert(WTN == 64 && WTM % 32 == 0, "wave tile");
  static_assert(kWaves >= kFW && BM % 64 == 0 && BN % 64 == 0, "fetches");
  static_assert(kSmem <= 160 * 1024 && (NS - 2) * (kLoadsA + kLoadsB) < 64, "LDS, vmcnt range");
  static_assert((!AK || BM >= 128) && (!BK || BN >= 128), "kn_off's key needs 16 chunks per k-row");
};

// An operand fragment of 32 rows for k step s of a slab: lane l holds 8
// consecutive k, from 16 s + 8 (l / 32) on, of row l % 32.
template <bool KM, int PITCH>
__device__ __forceinline__ bf16x8 ffn_frag(const char *st, int row0, int s, int lane) {
  if constexpr (KM) {
    const int g = lane >> 4, si = lane & 15;
    const int row = 16 * s + 8 * (g >> 1) + (si >> 2);
    const int col = row0 + 16 * (g & 1) + 4 * (si & 3);
    const int off = kn_off(row, col >> 3, PITCH) + 8 * (si & 1);
    const half4 lo = lds_read_tr16(st + off);
    const half4 hi = lds_read_tr16(st + off + 4 * PITCH);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    return *reinterpret_cast<const bf16x8 *>(st + swz(row0 + (lane & 31), 2 * s + (lane >> 5)));
  }
}

// The planes of pass i of an fp32 product, small terms first: A's plane in the
// low two bits, B's above.
__device__ __forceinline__ int plane_pair(int i) {
  // (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
  constexpr uint32_t t = 2u | (5u << 4) | (8u << 8) | (1u << 12) | (4u << 16) | (0u << 20);
  return int((t >> (4 * i)) & 15u);
}

// The corner of a product's tile t.
template <int BM, int BN, int EPI>
__device__ __forceinline__ void tile_corner(const FfnProb &p, int t, int &m0, int &n0) {
  int row, col;
  tile_place(t, p.tm, p.tn, row, col);
  m0 = row * BM;
  n0 = col * (EPI == kAct ? BN / 2 : BN);
}

// What becomes of 8 consecutive sums v of row `row` from column `col` on; kAct: of
// a's (v) and b's.
// kActBack: `kept`, a and b there.
template <bool F32>
struct KeptPair {
  KeptRaw<F32> a, b;
  __device__ __forceinline__ void load(const FfnArgs &args, int rows, int row, int col) {
    if (row < rows && col < args.ldf) {
      a.load(args.a, row, col);
      b.load(args.b, row, col);
    }
  }
};
template <int EPI, bool F32>
__device__ __forceinline__ void finish(const FfnArgs &args, const FfnProb &pr, int row, int col, float (&v)[8],
                                       float (&b)[8], const KeptPair<F32> &kept) {
  if (row >= pr.m) return;
  if constexpr (EPI == kStore) {
    if (col < pr.n) store_some<F32>(pr.out, int64_t(row) * pr.ldo + col, pr.n - col, v);
    return;
  }
  if (col >= args.ldf) return;
  const int64_t at = int64_t(row) * args.ldf + col;
  float h[8];
  if constexpr (EPI == kAct) {
    if (args.a.v) {
      store_kept<F32>(args.a, row, col, v);
      store_kept<F32>(args.b, row, col, b);
    }
    with_act(args.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float f, sl;
        act_and_slope<F32, decltype(act)::value>(v[j], f, sl);
        h[j] = f * b[j];
      }
    });
    store_planes<F32>(args.h + at * 2, args.plane, h);
  } else {
    with_act(args.act, [&](auto act) {
      auto one = [&](float a, float bj, float vj, float &hj, float &da, float &db) {
        float f, sl;
        act_and_slope<F32, decltype(act)::value>(a, f, sl);
        hj = f * bj;
        db = vj * f;
        da = vj * bj * sl;
      };
      if constexpr (F32) {
        float a[8], da[8], db[8];
        kept.a.values(a);
        kept.b.values(b);
#pragma unroll
        for (int j = 0; j < 8; ++j) one(a[j], b[j], v[j], h[j], da[j], db[j]);
        store_planes<true>(args.h + at * 2, args.plane, h);
        store_planes<true>(args.da + at * 2, args.plane, da);
        store_planes<true>(args.db + at * 2, args.plane, db);
      } else {
        // four values at a time, rounded before the next four: the registers hold the
        // sums and the next block's a and b as well
        bf16x4 o[3][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float4v r[3], a4, b4;
          kept.a.half(i, a4);
          kept.b.half(i, b4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x, y, z;
            one(a4[j], b4[j], v[4 * i + j], x, y, z);
            r[0][j] = x;
            r[1][j] = y;
            r[2][j] = z;
          }
#pragma unroll
          for (int q = 0; q < 3; ++q) o[q][i] = __builtin_convertvector(r[q], bf16x4);
          __builtin_amdgcn_sched_barrier(0);
        }
        char *const to[3] = {args.h, args.da, args.db};
#pragma unroll
        for (int q = 0; q < 3; ++q)
          *reinterpret_cast<bf16x8 *>(to[q] + at * 2) = __builtin_shufflevector(o[q][0], o[q][1], 0, 1, 2, 3, 4, 5, 6, 7);
      }
    });
  }
}

template <int BM, int BN, int WGM, int WGN, int NS, bool AK, bool BK, int EPI, bool F32>
__global__ __launch_bounds__(64 * WGM * WGN) void k_ffn(FfnArgs args) {
  using S = FfnTile<BM, BN, WGM, WGN, NS, AK, BK>;
  constexpr int FM = S::FM, FN = S::FN, FW = S::kFW;
  __shared__ __attribute__((aligned(16))) char smem[S::kSmem];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lr = lane & 31, lk = lane >> 5;
  const int wm = wave / WGN, wn = wave % WGN;

  // Block -> tile, or part of a tail tile: each XCD (block index modulo 8; `whole`
  // is a multiple of 8 where there is a tail) takes consecutive ones, in which 8
  // tiles of one column of tiles follow each other, so the blocks of an XCD share
  // operand panels in its L2.
  const bool part = int(blockIdx.x) >= args.whole;
  int tile, s0 = 0, s1 = args.slabs, slot = 0;
  if (part) {
    slot = by_xcd(int(blockIdx.x) - args.whole, args.tail * args.parts);
    part_place(slot, args.tail, args.per, args.slabs, tile, s0, s1);
    tile += args.whole;
  } else {
    tile = by_xcd(int(blockIdx.x), args.whole);
  }
  const int ns = s1 - s0;
  FfnProb pr = args.p[0];
  if (args.nprob > 1 && tile >= args.p[1].tile0) pr = args.p[1];
  if (args.nprob > 2 && tile >= args.p[2].tile0) pr = args.p[2];
  int m0, n0;
  tile_corner<BM, BN, EPI>(pr, tile - pr.tile0, m0, n0);
  // k: nsrc (times six passes) segments of nkt slabs; this block's slabs [s0, s1)
  const int nkt = (pr.k + 63) >> 6;
  const int kp = (pr.k + 7) & ~7;
  int seg = nkt ? s0 / nkt : 0, kt = s0 - seg * nkt;      // the next slab to fetch

  const uint32_t lds0 = lds_offset(smem);
  auto clamp31 = [](int64_t v) { return uint32_t(v < 0x7fffffff ? v : 0x7fffffff); };
  // N fetches of 8 rows each, row_step rows apart, to every FW-th (twice: 2 FW-th)
  // KB of the stage from `dst` on; `limit` valid rows from the first on
  auto fetch_rows = [&](auto n, auto lds_step, const char *base, int64_t ld, int64_t limit, int k0, uint32_t dst,
                        int row_step) {
    const i32x4 rs = buffer_rsrc(base + int64_t(k0) * 2, limit > 0 ? clamp31(((limit - 1) * ld + kp - k0) * 2) : 0u);
    const int row = wave * 8 + (lane >> 3), c = (lane & 7) ^ swz_key(row);
    uint32_t voff = (uint32_t(row) * uint32_t(ld) + uint32_t(c * 8)) * 2u;
    if (k0 + 64 > kp && k0 + c * 8 >= kp) voff = 0x80000000u;
    fetch_run<decltype(n)::value, decltype(lds_step)::value>(rs, voff, uint32_t(row_step) * uint32_t(ld) * 2u, dst + wave * 1024);
  };
  auto fetch_kn = [&](auto n, auto pitch_c, const char *base, int64_t ld, int k0, int cols, uint32_t dst) {
    constexpr int pitch = decltype(pitch_c)::value, cpr = pitch / 16, rpx = 1024 / pitch;
    const i32x4 rs = buffer_rsrc(base + int64_t(k0) * ld * 2, clamp31((int64_t(pr.k - k0 - 1) * ld + cols) * 2));
    const int row = wave * rpx + lane / cpr;
    const uint32_t voff = (uint32_t(row) * uint32_t(ld) + uint32_t(((lane % cpr) ^ ((row & 3) << 2)) * 8)) * 2u;
    fetch_run<decltype(n)::value, FW * 1024>(rs, voff, uint32_t(rpx * FW) * uint32_t(ld) * 2u, dst + wave * 1024);
  };
  constexpr std::integral_constant<int, S::kLoadsA> nA{};
  constexpr std::integral_constant<int, S::kLoadsB> nB{};
  constexpr std::integral_constant<int, S::kLoadsB / 2> nHalf{};
  constexpr std::integral_constant<int, FW * 1024> each{};
  constexpr std::integral_constant<int, 2 * FW * 1024> other{};
  constexpr std::integral_constant<int, BM * 2> pitchA{};
  constexpr std::integral_constant<int, BN * 2> pitchB{};
  auto dload = [&](int st) {
    const int src = pr.nsrc > 1 ? seg & 1 : 0;
    int64_t oa = 0, ob = 0;
    if constexpr (F32) {
      const int pp = plane_pair(pr.nsrc > 1 ? seg >> 1 : seg);
      oa = (pp & 3) * pr.pa;
      ob = (pp >> 2) * pr.pb;
    }
    const int k0 = kt * 64;
    if (++kt == nkt) {
      kt = 0;
      ++seg;
    }
    if (wave >= FW) return;
    const uint32_t sA = lds0 + uint32_t(st) * S::kStage, sB = sA + S::kStageA;
    const char *A = pr.a[0] + oa, *B = pr.b[0] + ob;
    if (src) {
      A = pr.a[1] + oa;
      B = pr.b[1] + ob;
    }
    if constexpr (AK) fetch_kn(nA, pitchA, A + int64_t(m0) * 2, pr.lda, k0, ((pr.m + 7) & ~7) - m0, sA);
    else fetch_rows(nA, each, A + int64_t(m0) * pr.lda * 2, pr.lda, pr.m - m0, k0, sA, 8 * FW);
    if constexpr (BK) {
      fetch_kn(nB, pitchB, B + int64_t(n0) * 2, pr.ldb, k0, ((pr.n + 7) & ~7) - n0, sB);
    } else if constexpr (EPI == kAct) {
      // rows 64 w .. 64 w + 31 of the stage: Wg's rows n0 + 32 w .., the next 32: Wu's
      static_assert(FW == 4, "32 rows per half");
      fetch_rows(nHalf, other, B + int64_t(n0) * pr.ldb * 2, pr.ldb, pr.n - n0, k0, sB, 32);
      fetch_rows(nHalf, other, pr.b[1] + ob + int64_t(n0) * pr.ldb * 2, pr.ldb, pr.n - n0, k0, sB + FW * 1024, 32);
    } else {
      fetch_rows(nB, each, B + int64_t(n0) * pr.ldb * 2, pr.ldb, pr.n - n0, k0, sB, 8 * FW);
    }
  };

  floatx16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  // kActBack: a and b of a 32-row block of the wave tile are loaded a block ahead,
  // the first ones before the products (fp32 tensors: with the block, there are
  // no registers for more)
  constexpr int PC = EPI == kAct ? 4 : 8;                 // 8-column pieces per row
  constexpr int kTasks = 32 * PC / 64;
  constexpr bool kAhead = EPI == kActBack && !F32;
  KeptPair<F32> kept[kAhead ? kTasks : 1];
  auto kept_load = [&](int i, int t) {
    const int task = lane + 64 * t;
    kept[t].load(args, pr.m, m0 + wm * S::WTM + i * 32 + task / PC, n0 + wn * 64 + (task % PC) * 8);
  };
  if constexpr (kAhead) {
    if (!part) {
#pragma unroll
      for (int t = 0; t < kTasks; ++t) kept_load(0, t);
    }
  }

#pragma unroll
  for (int q = 0; q < NS - 1; ++q)
    if (q < ns) dload(q);
  for (int it = 0, st = 0; it < ns; ++it, st = st + 1 == NS ? 0 : st + 1) {
    vm_wait_slabs<S::kLoadsA + S::kLoadsB, NS - 2>(min(NS - 2, ns - 1 - it));
    __syncthreads();                 // slab `it` is published; the one before it is done
    if (it + NS - 1 < ns) dload(st == 0 ? NS - 1 : st - 1);
    const char *sA = smem + st * S::kStage, *sB = sA + S::kStageA;
    bf16x8 fa[2][FM], fb[2][FN];
    auto read = [&](int s, int slot) {
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[slot][i] = ffn_frag<AK, BM * 2>(sA, wm * S::WTM + i * 32, s, lane);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[slot][j] = ffn_frag<BK, BN * 2>(sB, wn * S::WTN + j * 32, s, lane);
    };
    read(0, 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) read(s + 1, (s + 1) & 1);
      // operands swapped: acc[i][j][4 g + q] = C[row lr of block i][column 32 j + 8 g + 4 lk + q]
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][j], fa[s & 1][i], acc[i][j], 0, 0, 0);
    }
    // the first k step's reads, then each step's MFMAs with the next step's
    // reads spread among them
    constexpr int kReads = FM * (AK ? 2 : 1) + FN * (BK ? 2 : 1), kMfma = FM * FN;
    constexpr int kGroups = kReads < kMfma ? kReads : kMfma;
    __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        __builtin_amdgcn_sched_group_barrier(0x008, kMfma / kGroups, 0);
        if (s < 3) __builtin_amdgcn_sched_group_barrier(0x100, kReads / kGroups, 0);
      }
  }
  __syncthreads();                   // the epilogue reuses the stages

  // Epilogue, per 32-row block of the wave tile: the fp32 sums go through the
  // wave's own LDS area (one wave's LDS operations keep their order, so a
  // wave-level barrier suffices), then each lane takes 8 consecutive columns.
  float *ef = reinterpret_cast<float *>(smem) + wave * 32 * S::kPitch;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4v *>(ef + lr * S::kPitch + 32 * j + 8 * g + 4 * lk) =
            float4v{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    __builtin_amdgcn_wave_barrier();
    const int row0 = wm * S::WTM + i * 32;
    constexpr int kCopies = F32 && EPI != kStore ? 1 : kTasks;   // fp32 activations are long code
#pragma unroll kCopies
    for (int t = 0; t < kTasks; ++t) {
      const int task = lane + 64 * t, rl = task / PC, cl = (task % PC) * 8;
      float v[8], b[8];
      auto staged = [&](int c, float (&o)[8]) {
        const float4v e0 = *reinterpret_cast<const float4v *>(ef + rl * S::kPitch + c);
        const float4v e1 = *reinterpret_cast<const float4v *>(ef + rl * S::kPitch + c + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = j < 4 ? e0[j & 3] : e1[j & 3];
      };
      staged(cl, v);
      if constexpr (EPI == kAct) staged(32 + cl, b);
      if (part) {
        const int64_t at = (int64_t(slot) * BM + row0 + rl) * BN + wn * 64 + cl;
        store_whole<true>(args.part, at, v);
        if constexpr (EPI == kAct) store_whole<true>(args.part, at + 32, b);
      } else {
        KeptPair<F32> k;
        if constexpr (kAhead) k = kept[t];
        else if constexpr (EPI == kActBack) k.load(args, pr.m, m0 + row0 + rl, n0 + wn * 64 + cl);
        finish<EPI, F32>(args, pr, m0 + row0 + rl, n0 + wn * (EPI == kAct ? 32 : 64) + cl, v, b, k);
        if constexpr (kAhead) {
          if (i + 1 < FM) kept_load(i + 1, t);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The sums of a tail tile's parts, in the order of k, and what becomes of them: a
// thread 8 columns. HBM and latency (125 MB in 20 us, 6 TB/s; small tails 4-5 us).
template <int BM, int BN, int EPI, bool F32>
__global__ __launch_bounds__(256) void k_tail(FfnArgs args) {
  constexpr int PC = EPI == kAct ? BN / 16 : BN / 8;      // pieces per tile row
  const int tt = blockIdx.y, tile = args.whole + tt;
  FfnProb pr = args.p[0];
  if (args.nprob > 1 && tile >= args.p[1].tile0) pr = args.p[1];
  if (args.nprob > 2 && tile >= args.p[2].tile0) pr = args.p[2];
  int m0, n0;
  tile_corner<BM, BN, EPI>(pr, tile - pr.tile0, m0, n0);
  const int task = int(blockIdx.x) * 256 + threadIdx.x, row = task / PC, q = task % PC;
  if (row >= BM || m0 + row >= pr.m) return;
  // kAct: piece q is columns 8 q of h; its a and b sums lie 32 columns apart
  const int col = EPI == kAct ? (q >> 2) * 64 + (q & 3) * 8 : q * 8;
  float v[8] = {}, b[8] = {};
  for (int c = 0; c < args.parts; ++c) {
    const int64_t at = ((int64_t(c) * args.tail + tt) * BM + row) * BN + col;
    float w[8];
    load_whole<true>(args.part, at, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
    if constexpr (EPI == kAct) {
      load_whole<true>(args.part, at + 32, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] += w[j];
    }
  }
  KeptPair<F32> kept;
  if constexpr (EPI == kActBack) kept.load(args, pr.m, m0 + row, n0 + q * 8);
  finish<EPI, F32>(args, pr, m0 + row, n0 + q * 8, v, b, kept);
}

// ---------------------------------------------------------------------------
// The forward products for a few tokens (TF x 16 at most), whose time is the
// reading of the weights: a block takes 16 rows of each weight (DUAL: of Wg and
// Wu) and its waves share k in chunks of 128 bytes per row; a lane's 16 bytes of
// a weight row go from memory to the matrix instruction's operand as they are
// (lane l: row l % 16, k from 8 (l / 16) on; fp32: four k of 4 (l / 16) on in
// four instructions), the tokens are the other operand, read through the caches
// by every block. The waves' sums meet in LDS. No row alignment is needed. One token
// of 1536 x 6144 in bf16: 38 MB of Wg and Wu in 11.1 us, 19 MB of Wd in 9.1, where the
// copy's rate would take 7.7 and 3.9. Blocks bound it where there are fewer than CUs: 384
// read Wg and Wu, but 96 read Wd, and 160 of the 256 CUs read nothing meanwhile (7 tokens
// of 768 x 2048 in fp32: 128 and 48 blocks, 7.7 and 8.1 us). The rest is the start of a
// launch, one trip to HBM and the sums' way through LDS. The tiles of k_ffn take 33 us for
// both launches. Not kept: chunks loaded one to three ahead (19.0 against 18.6 us), blocks
// that begin at different chunks (no change).
struct FewArgs {
  const void *x, *w0, *w1;
  void *out;                   // h or y
  int64_t ldx, ldo;
  int32_t tokens, n, k, act;
};

template <int TF, bool DUAL, bool F32>
__global__ __launch_bounds__(TF > 2 ? 512 : 1024) void k_few(FewArgs a) {
  using T = typename std::conditional<F32, float, uint16_t>::type;
  constexpr int NF = DUAL ? 2 : 1, kWaves = TF > 2 ? 8 : 16;
  constexpr int kChunk = F32 ? 32 : 64;                // k per chunk of 128 bytes
  constexpr int kLane = F32 ? 4 : 8, kStep = 4 * kLane;
  __shared__ float4v red[kWaves][NF * TF][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = int(blockDim.x) >> 6;
  const int n0 = int(blockIdx.x) * 16, r = lane & 15, kl = (lane >> 4) * kLane;
  // rows past the end read the last one again; their results go nowhere
  const int64_t wrow = int64_t(min(n0 + r, a.n - 1)) * a.k;
  const T *w[NF], *x[TF];
  w[0] = static_cast<const T *>(a.w0) + wrow;
  if constexpr (DUAL) w[NF - 1] = static_cast<const T *>(a.w1) + wrow;
#pragma unroll
  for (int t = 0; t < TF; ++t) x[t] = static_cast<const T *>(a.x) + int64_t(min(16 * t + r, a.tokens - 1)) * a.ldx;
  float4v acc[NF][TF];
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int t = 0; t < TF; ++t) acc[i][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

  auto load = [&](const T *row, int k) {
    if constexpr (F32) {
      if (k + 4 <= a.k) return *(const SLORR_GLOBAL u32x4_any *)(row + k);
      u32x4_any v{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (k + j < a.k) v[j] = __float_as_uint(row[k + j]);
      return v;
    } else {
      return get(row, k, a.k).q[0];
    }
  };
  struct Chunk {
    u32x4 w[2][NF], x[2][TF];
  } c;
  auto whole = [](const T *row, int k) { return u32x4(*(const SLORR_GLOBAL u32x4_any *)(row + k)); };
  auto fetch = [&](int k, auto get) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < NF; ++i) c.w[s][i] = get(w[i], k + s * kStep + kl);
#pragma unroll
      for (int t = 0; t < TF; ++t) c.x[s][t] = get(x[t], k + s * kStep + kl);
    }
  };
  auto multiply = [&]() {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int t = 0; t < TF; ++t) {
          if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c.w[s][i][j]), __uint_as_float(c.x[s][t][j]),
                                                               acc[i][t], 0, 0, 0);
          } else {
            acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, c.w[s][i]),
                                                                __builtin_bit_cast(bf16x8, c.x[s][t]), acc[i][t], 0, 0, 0);
          }
        }
  };
  // whole chunks without the code for a row's end, then that end by the wave whose
  // turn it is
  for (int k = wave * kChunk; k + kChunk <= a.k; k += waves * kChunk) {
    fetch(k, whole);
    multiply();
  }
  const int end = a.k / kChunk;
  if (end * kChunk < a.k && end % waves == wave) {
    fetch(end * kChunk, load);
    multiply();
  }
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int t = 0; t < TF; ++t) red[wave][i * TF + t][lane] = acc[i][t];
  __syncthreads();
  // lane l of result block t: token 16 t + l % 16, rows 4 (l / 16) .. + 3
  for (int t = wave; t < TF; t += waves) {
    float4v s[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      s[i] = red[0][i * TF + t][lane];
      for (int q = 1; q < waves; ++q) s[i] += red[q][i * TF + t][lane];
    }
    const int token = 16 * t + r, n = n0 + 4 * (lane >> 4);
    if (token >= a.tokens) continue;
    T *o = static_cast<T *>(a.out) + token * a.ldo + n;
    if constexpr (DUAL) {
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float f, slope;
          act_and_slope<F32, decltype(act)::value>(s[0][j], f, slope);
          s[0][j] = f * s[NF - 1][j];
        }
      });
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < a.n) o[j] = from_f<T>(s[0][j]);
  }
}

}  // namespace slorr
