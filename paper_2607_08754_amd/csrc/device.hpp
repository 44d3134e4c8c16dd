// Device helpers that the library's kernels share: types and conversions, 16-byte
// accesses, LDS layouts, direct global -> LDS fetches and their waits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace slorr {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint16_t bf16_t;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return __uint_as_float(uint32_t(v) << 16); }
__device__ __forceinline__ float to_f(_Float16 v) { return float(v); }

// fp32 -> bf16 with round to nearest, ties to even (a NaN stays a quiet NaN):
// add half an ulp of the bf16 result, minus one when the kept part is even,
// then truncate.
__device__ __forceinline__ bf16_t f32_to_bf16(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return bf16_t((u >> 16) | 0x40u);
  u += 0x7fffu + ((u >> 16) & 1u);
  return bf16_t(u >> 16);
}

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ _Float16 from_f<_Float16>(float v) { return _Float16(v); }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float v) { return f32_to_bf16(v); }

// The full-tile path of the tile kernels below: 16-byte accesses known to be
// aligned and in bounds, issued as global-memory instructions with no branch
// between them, so that all of a thread's loads are in flight together (the
// weight and gradient pointers come from a device table: left to itself the
// compiler cannot tell their address space and emits flat accesses).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 gload16(const void *p) {
  return *(const __attribute__((address_space(1))) u32x4 *)p;
}
__device__ __forceinline__ void gstore16(void *p, u32x4 v) { *(__attribute__((address_space(1))) u32x4 *)p = v; }
__device__ __forceinline__ u32x4 gload16_stream(const void *p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4 *)p);
}

// 8 consecutive values as loaded. Rows need no 16-byte alignment: the memory
// system takes 16-byte accesses at any multiple of the element.
template <typename T>
struct Raw {
  u32x4 q[sizeof(T) / 2];
};
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
#define SLORR_GLOBAL __attribute__((address_space(1)))

// The end of a row, n < 8 values, goes as runs of 4, 2 and 1: three accesses with
// one address between them (a load and a store per value cost these kernels 50
// registers, and with them half of their waves).
template <typename T>
__device__ __forceinline__ Raw<T> get(const T *row, int c, int dim) {
  Raw<T> r;
  if (c + 8 <= dim) {
    const SLORR_GLOBAL u32x4_any *p = (const SLORR_GLOBAL u32x4_any *)(row + c);
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) r.q[i] = p[i];
    return r;
  }
#pragma unroll
  for (int i = 0; i < int(sizeof(T) / 2); ++i) r.q[i] = u32x4{0, 0, 0, 0};
  const int n = dim - c;
  if (n <= 0) return r;
  const bool h4 = n & 4, h2 = n & 2;
  const T *p2 = row + c + (n & 4), *p1 = row + c + (n & 6);
  if constexpr (sizeof(T) == 2) {
    u32x2_any a{0, 0};
    uint32_t b = 0, d = 0;
    if (h4) a = *(const SLORR_GLOBAL u32x2_any *)(row + c);
    if (h2) b = *(const SLORR_GLOBAL u32_any *)p2;
    if (n & 1) d = *(const SLORR_GLOBAL uint16_t *)p1;
    const uint32_t lo = h2 ? b : d, hi = h2 ? d : 0u;
    r.q[0] = u32x4{h4 ? a[0] : lo, h4 ? a[1] : hi, h4 ? lo : 0u, h4 ? hi : 0u};
  } else {
    u32x4 a{0, 0, 0, 0};
    u32x2_any b{0, 0};
    uint32_t d = 0;
    if (h4) a = *(const SLORR_GLOBAL u32x4_any *)(row + c);
    if (h2) b = *(const SLORR_GLOBAL u32x2_any *)p2;
    if (n & 1) d = *(const SLORR_GLOBAL u32_any *)p1;
    const uint32_t e0 = h2 ? b[0] : d, e1 = h2 ? b[1] : 0u, e2 = h2 ? d : 0u;
    r.q[0] = h4 ? a : u32x4{e0, e1, e2, 0u};
    if (h4) r.q[sizeof(T) / 2 - 1] = u32x4{e0, e1, e2, 0u};
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void widen(const Raw<T> &r, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 2) v[j] = __uint_as_float(j & 1 ? r.q[0][j >> 1] & 0xffff0000u : r.q[0][j >> 1] << 16);
    else v[j] = __uint_as_float(r.q[j >> 2][j & 3]);
  }
}

// Byte offset of 16-byte chunk `chunk` of LDS row `row`. The XOR key
// (row & 7) ^ ((row >> 3) & 1) permutes the chunks so that (a) any 8
// consecutive rows (one 8-lane phase of a 16-byte read with 32 banks) use 8
// distinct chunk positions, and (b) any 16 consecutive rows (a 16-lane phase
// with 64 banks, where rows of equal parity share a 128-byte bank half) use 8
// distinct positions per parity.
__device__ __forceinline__ int swz_key(int row) { return (row & 7) ^ ((row >> 3) & 1); }
__device__ __forceinline__ int swz(int row, int chunk) { return row * 128 + ((chunk ^ swz_key(row)) << 4); }

// 16 bytes per lane from a buffer straight into LDS: byte voff + soff of the
// buffer (voff per lane, soff wave-uniform) lands at lds_base + 16 l
// (lds_base wave-uniform, passed in m0). On the update tile's k loop this
// form issues at a markedly lower cost than global_load_lds_dwordx4 with a
// 64-bit address per lane; a load past the buffer's size returns zeros
// instead of faulting. Device pass only: the host pass of the single-source
// build just needs the kernel's stub.
//
// Issued through inline assembly: the compiler then does not track these LDS
// writes and puts no wait for them before later LDS reads (it cannot tell
// that those read the other stage). Completion is the caller's job: each
// k-slab is waited for by count (s_waitcnt vmcnt) before the block barrier
// that publishes it.
//
// The compiler does not see a memory instruction in the assembly either, and so
// keeps none of the distances that one needs: one wait state after m0 was
// written, and five after a vector instruction wrote one of its scalar registers.
// WAIT + 1 of them stand here: 0 where the operands come from scalar
// instructions, 4 where v_readfirstlane may have written them. Kernels with more
// scalar values than registers, where v_readlane can come right before a fetch,
// use fetch_run below.
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 buffer_rsrc(const void *base, uint32_t bytes) {
  const uint64_t b = uint64_t(uintptr_t(base));
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane(int(uint32_t(b)));
  r[1] = __builtin_amdgcn_readfirstlane(int(uint32_t(b >> 32) & 0xffffu));   // stride 0
  r[2] = __builtin_amdgcn_readfirstlane(int(bytes));                        // size in bytes
  r[3] = 0x00020000;                                                         // raw 32-bit dwords
  return r;
}
template <int WAIT = 0>
__device__ __forceinline__ void buffer_load_lds16(i32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t m = __builtin_amdgcn_readfirstlane(lds_base);
  const uint32_t so = __builtin_amdgcn_readfirstlane(soff);
  asm volatile("s_nop %4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "{m0}"(m), "v"(voff), "s"(rsrc), "s"(so), "n"(WAIT) : "memory");
#else
  (void)rsrc;
  (void)voff;
  (void)soff;
  (void)lds_base;
#endif
}
__device__ __forceinline__ void buffer_load_lds16(i32x4 rsrc, uint32_t voff, uint32_t soff, void *lds_base) {
  buffer_load_lds16(rsrc, voff, soff, uint32_t(uintptr_t(lds_base)));
}

// N fetches in a row (see buffer_load_lds16): fetch i takes byte voff + i soff_step
// of the buffer to lds_base + i kLdsStep + 16 l. One block of assembly, which keeps
// its own distances: five wait states ahead of the first fetch for the operands'
// sake (without them fetches took an operand's old value where the compiler's
// v_readlane came right before: an fp32 product of 4 x 64 x 64 was off by 3e-6 now
// and then), and one between each write of m0 and its fetch.
template <int N, int kLdsStep>
__device__ __forceinline__ void fetch_run(i32x4 rsrc, uint32_t voff, uint32_t soff_step, uint32_t lds_base) {
  static_assert(N == 2 || N == 4 || N == 8, "fetches in a row");
#if defined(__HIP_DEVICE_COMPILE__)
  uint32_t m = __builtin_amdgcn_readfirstlane(lds_base), so = 0;
  const uint32_t step = __builtin_amdgcn_readfirstlane(soff_step);
#define SLORR_FETCH "buffer_load_dwordx4 %2, %3, %0 offen lds\n\t"
#define SLORR_NEXT "s_add_u32 m0, m0, %5\n\ts_add_u32 %0, %0, %4\n\t" SLORR_FETCH
#define SLORR_FIRST "s_nop 4\n\t" SLORR_FETCH
  if constexpr (N == 2)
    asm volatile(SLORR_FIRST SLORR_NEXT : "+&s"(so), "+{m0}"(m) : "v"(voff), "s"(rsrc), "s"(step), "n"(kLdsStep) : "memory", "scc");
  else if constexpr (N == 4)
    asm volatile(SLORR_FIRST SLORR_NEXT SLORR_NEXT SLORR_NEXT
                 : "+&s"(so), "+{m0}"(m) : "v"(voff), "s"(rsrc), "s"(step), "n"(kLdsStep) : "memory", "scc");
  else
    asm volatile(SLORR_FIRST SLORR_NEXT SLORR_NEXT SLORR_NEXT SLORR_NEXT SLORR_NEXT SLORR_NEXT SLORR_NEXT
                 : "+&s"(so), "+{m0}"(m) : "v"(voff), "s"(rsrc), "s"(step), "n"(kLdsStep) : "memory", "scc");
#undef SLORR_FETCH
#undef SLORR_NEXT
#undef SLORR_FIRST
#else
  (void)rsrc;
  (void)voff;
  (void)soff_step;
  (void)lds_base;
#endif
}

// Transposing LDS read of 16-bit values (ds_read_b64_tr_b16). Within each
// group of 16 lanes, lane s gives the address of 4 consecutive values: row
// s / 4, columns 4 (s % 4) .. 4 (s % 4) + 3 of a 4 x 16 block; lane j then
// holds column j of the block, element i from row i.
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ half4 lds_read_tr16(const void *lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((__vector_size__(4 * sizeof(__fp16)))) __fp16 fp16x4;
  typedef __attribute__((address_space(3))) fp16x4 lds_fp16x4;
  const fp16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_fp16x4 *)(lds));
  return __builtin_bit_cast(half4, v);
#else
  (void)lds;
  return half4{};
#endif
}

// Byte offset of 16-byte chunk `chunk` of k-row `row`
// of a [k][n] operand stage (rows of `pitch` bytes). The key 4 (row & 3)
// spreads the 4 rows x 4 chunks that one half-wave reads with a transposing
// read (rows r..r+3 of a 16-row step, 64 bytes each) over all 64 banks.
__device__ __forceinline__ int kn_off(int row, int chunk, int pitch) {
  return row * pitch + ((chunk ^ ((row & 3) << 2)) << 4);
}

// LDS byte offset of a shared array. The fetches below take offsets, not
// pointers: a generic pointer would be cast back to LDS with a null check.
__device__ __forceinline__ uint32_t lds_offset(const char *smem) {
#if defined(__HIP_DEVICE_COMPILE__)
  return uint32_t(uintptr_t((const __attribute__((address_space(3))) char *)smem));
#else
  (void)smem;
  return 0;
#endif
}

// s_waitcnt vmcnt(N), the other counters left alone (gfx9 encoding).
template <int N>
__device__ __forceinline__ void vm_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// Wait until at most `ahead` (<= A) slabs of fetches, L instructions each,
// issued by this wave are outstanding.
template <int L, int A>
__device__ __forceinline__ void vm_wait_slabs(int ahead) {
  if constexpr (A >= 2) {
    if (ahead >= 2) {
      vm_wait<2 * L>();
      return;
    }
  }
  if constexpr (A >= 1) {
    if (ahead >= 1) {
      vm_wait<L>();
      return;
    }
  }
  vm_wait<0>();
}

}  // namespace slorr
