// What the kernels of the 4-bit paged cache share: the tile layout, checks of the cache.
#pragma once
#include "kvd_q8.h"

namespace kvd {
namespace q4 {

using q8::kTile;
using q8::aligned;
using q8::launched;
using q8::pack2;
using q8::stride_ok;
using q8::two_to;
typedef q8::f32x2 f32x2;
typedef q8::f32x4 f32x4;

constexpr int kBlock = 32;                     // elements of a scale
constexpr int kValues = 1024, kKeyScales = 2048, kValueScales = 2112;    // where they begin in a tile
constexpr int kTileBytes = 2176;               // seventeen lines of 128 bytes
constexpr int kExpMin = -96, kExpMax = 125;    // exponents of a scale
constexpr int kBias = 127;

inline int check_cache(const kvd_q4_cache* c, const kvd_q8_rows* r) {
  if (!c) return KVD_ERR_ARG;
  if (int e = q8::check_rows(r)) return e;
  if (c->kv_dtype != KVD_F16 && c->kv_dtype != KVD_BF16) return KVD_ERR_DTYPE;
  if (c->head_dim != kHeadDim || c->page_size != r->page_size || c->n_blocks != r->n_blocks) return KVD_ERR_SHAPE;
  if (c->n_kv_heads < 1 || c->n_kv_heads > q8::kMaxHeads || c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads) return KVD_ERR_SHAPE;
  if (c->n_q_heads / c->n_kv_heads > KVD_MAX_GROUP) return KVD_ERR_SHAPE;
  // tiles are addressed by a line's number in 32 bits
  if ((int64_t)c->n_blocks * c->n_kv_heads * (c->page_size / kTile) * (kTileBytes / 128) >= (int64_t)UINT32_MAX) return KVD_ERR_SHAPE;
  if (!(c->softmax_scale >= 0.f) || isinf(c->softmax_scale)) return KVD_ERR_ARG;
  return KVD_OK;
}

}  // namespace q4
}  // namespace kvd
