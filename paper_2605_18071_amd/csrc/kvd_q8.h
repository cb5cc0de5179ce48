// What the kernels of the 8-bit paged cache share: the tile layout, conversions, checks of the two structs.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "kvd_device.h"
#include "kvd_internal.h"

namespace kvd {
namespace q8 {

constexpr int kTile = 16;                      // tokens of a tile
constexpr int kHalfTile = kTile * kHeadDim;    // bytes of a tile's keys, and of its values behind them
constexpr int kTileBytes = 2 * kHalfTile;
constexpr int kExpMin = -96;                   // least exponent of a scale: everything below 2^-105 is 0
// What a workspace begins with: the attention's tickets, zero between calls.  The scores of a selection lie behind them, so that
// one workspace may serve both calls, one after the other.
constexpr int kTicketBytes = 8192;
constexpr int kMaxSeqs = 4096, kMaxRows = 131072, kMaxHeads = 256, kMaxTablePages = 65536;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// 2^e as fp32, e in -126..127
__device__ __forceinline__ float two_to(int e) { return as_f32((u32)(e + 127) << 23); }

// Place of token t's element d in a tile: keys, and values (without their offset of kHalfTile)
__device__ __forceinline__ int key_at(int t, int d) { return (d >> 6) * 1024 + (((d >> 3) & 3) * 16 + t) * 16 + ((d >> 5) & 1) * 8 + (d & 7); }
__device__ __forceinline__ int value_at(int t, int d) { return (d >> 6) * 1024 + ((t >> 2) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (t & 3); }

// fp32 pair -> 16-bit pair, round to nearest even
template <bool BF16>
__device__ __forceinline__ u32 pack2(float a, float b) {
  const f32x2 v = {a, b};
  if (BF16) return __builtin_bit_cast(u32, __builtin_convertvector(v, bf16x2));
  return __builtin_bit_cast(u32, __builtin_convertvector(v, f16x2));
}

// The conditions that every call puts on the structs; n_blocks and page_size have to agree where both are given.
inline int check_rows(const kvd_q8_rows* r) {
  if (!r) return KVD_ERR_ARG;
  if (r->page_size < kTile || r->page_size > KVD_MAX_PAGE || r->page_size % kTile) return KVD_ERR_SHAPE;
  if (r->n_seqs < 1 || r->n_seqs > kMaxSeqs || r->max_pages < 1 || r->max_pages > kMaxTablePages) return KVD_ERR_SHAPE;
  if (r->n_rows < 1 || r->n_rows > kMaxRows || r->max_runs < 1 || r->max_runs > kMaxRows || r->n_blocks < 1) return KVD_ERR_SHAPE;
  return KVD_OK;
}
inline int check_cache(const kvd_q8_cache* c, const kvd_q8_rows* r) {
  if (!c) return KVD_ERR_ARG;
  if (int e = check_rows(r)) return e;
  if (c->kv_dtype != KVD_F16 && c->kv_dtype != KVD_BF16) return KVD_ERR_DTYPE;
  if (c->head_dim != kHeadDim || c->page_size != r->page_size || c->n_blocks != r->n_blocks) return KVD_ERR_SHAPE;
  if (c->n_kv_heads < 1 || c->n_kv_heads > kMaxHeads || c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads) return KVD_ERR_SHAPE;
  if (c->n_q_heads / c->n_kv_heads > KVD_MAX_GROUP) return KVD_ERR_SHAPE;
  if (c->sink_pages < 0 || c->recent_pages < 0) return KVD_ERR_SHAPE;
  if (!(c->softmax_scale >= 0.f) || isinf(c->softmax_scale)) return KVD_ERR_ARG;
  return KVD_OK;
}
inline bool aligned(const void* p, size_t n) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool stride_ok(int64_t stride, int heads) { return stride >= (int64_t)heads * kHeadDim && stride % 8 == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? KVD_OK : KVD_ERR_HIP; }

}  // namespace q8
}  // namespace kvd
