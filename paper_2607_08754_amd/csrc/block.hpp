// Host side of the operators of a regularised block (gated feed-forward, the
// join between blocks, dropout): argument checks' limits, workspace layouts and
// the enqueue entries (internal).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "kernels.hpp"
#include "slorr.h"

namespace slorr {

// Operand rows of the products are read in 16-byte chunks of 8 bf16 numbers:
// an operand whose rows are not 16-byte aligned is copied into the workspace
// with its row padded to a multiple of 8, the padding zero. An fp32 operand is
// held as three bf16 numbers per value (planes), in three such copies.
constexpr int64_t kMaxWidth = int64_t(1) << 20;      // dim, inner
constexpr int64_t kMaxStride = (int64_t(1) << 22) - 8;   // row strides, in elements: the 256 rows
                                                     // of a tile stay within 2 GiB
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1024;
// Forward alone: k_few up to 64 tokens, in bf16 beyond 16 while tokens * dim * inner
// stays below kFewWork: it reads the tokens in every block, k_ffn's tiles do not (us
// of k_few and k_ffn in bf16: 32 tokens of 1536 x 6144 33.7, 34.6, 64 of them 50, 35;
// 64 of 1280 x 3456 29.0, 29.2; 16 of 4096 x 11008 62, 71, 24 of them 75, 71; in
// fp32 64 of 4096 x 11008 285, 596).
constexpr int kFewTokens = 64;
constexpr int64_t kFewWork = 300000000;
constexpr int kMaxNorm = 8192;                       // dim of a join: 512 threads, two pieces of 8 each

inline int64_t up8(int64_t n) { return (n + 7) & ~int64_t(7); }

struct FfnShape {
  int64_t tokens, ldx, lddy;
  int32_t dim, inner, dtype, act;
  int planes() const { return dtype == SLORR_F32 ? 3 : 1; }
  size_t elem() const { return dtype == SLORR_F32 ? 4 : 2; }
  int64_t ldf() const { return up8(inner); }         // rows of the inner tensors
  int64_t ldd() const { return up8(dim); }
  bool few() const {
    return tokens <= kFewTokens && (dtype == SLORR_F32 || tokens <= 16 || tokens * dim * inner <= kFewWork);
  }
  // operands that are read in place: bf16 rows of whole chunks
  bool direct(int64_t width, int64_t ld) const { return dtype == SLORR_BF16 && width % 8 == 0 && ld % 8 == 0; }
};

constexpr size_t kAbsent = ~size_t(0);

// Byte offsets in a call's workspace; kAbsent: the operand is read in place.
struct FfnLayout {
  size_t x = kAbsent, dy = kAbsent, wg = kAbsent, wu = kAbsent, wd = kAbsent;
  size_t h = kAbsent, da = kAbsent, db = kAbsent;
  size_t part = kAbsent;       // fp32 partials of split products
  size_t bytes = 0;
};

FfnLayout ffn_layout(const FfnShape &s, bool backward);
size_t ffn_state_bytes(const FfnShape &s);

void enqueue_ffn_forward(const FfnShape &s, const void *x, const void *wg, const void *wu, const void *wd, void *y,
                         void *state, void *ws, hipStream_t st);
void enqueue_ffn_backward(const FfnShape &s, const void *dy, const void *x, const void *wg, const void *wu,
                          const void *wd, const void *state, void *dx, void *dwg, void *dwu, void *dwd, void *ws,
                          hipStream_t st);

struct JoinShape {
  int64_t rows, ldx, ldf, ld_gate, gate_rows;
  int32_t dim, dtype;
  int layer, post, pre;
  float eps, alpha;
  uint32_t drop;               // an element is dropped where its 16-bit number is below this
  int64_t site;
};

// How the backward pass cuts its rows into blocks (see k_join_bwd).
struct JoinCut {
  int64_t groups = 1, rows_per_group = 0;    // gate rows with a sum over tokens; one group without
  int64_t groups_per_block = 1, parts = 1, rows_per_part = 0;
  int64_t blocks = 0;
};
JoinCut join_cut(const JoinShape &s);
size_t join_workspace(const JoinShape &s);

void enqueue_join_forward(const JoinShape &s, const slorr_join_tensors_t &t, const int64_t *rng, void *y, void *z,
                          hipStream_t st);
void enqueue_join_backward(const JoinShape &s, const slorr_join_tensors_t &t, const int64_t *rng, const void *dy,
                           const void *dz, const slorr_join_grads_t &g, void *ws, hipStream_t st);

void enqueue_dropout(int64_t n, int32_t dtype, uint32_t drop, const int64_t *rng, int64_t site, const void *x,
                     void *y, hipStream_t st);

}  // namespace slorr
