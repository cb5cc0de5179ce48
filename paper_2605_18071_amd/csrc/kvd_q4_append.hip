// Writing a step's keys and values into the 4-bit pages, and reading them back.
//
// A token's 32 elements have a scale 2^e of their own, e the least with amax <= 7 * 2^e: the largest element then is off by
// no more than any other may be (a half step, as 6 is the last code), and the others have steps as fine as that allows.
// The hardware's conversion divides by the scale and rounds to nearest even, saturating at 6; nothing else rounds.
#include "kvd_q4.h"

namespace kvd {
namespace q4 {

constexpr int kAppendThreads = 256;            // 16 tokens x 16 lanes of 8 elements

struct AppendArgs {
  const uint16_t *k, *v;
  long long k_stride, v_stride;
  const int4* runs;
  unsigned char* pages;
  int H, P, NB, T;
};

// Exponent for the largest finite magnitude of 32 elements.  (7 = 0.875 * 2^3)
__device__ __forceinline__ int exp_for(float amax) {
  int x;
  const float m = frexpf(amax, &x);            // m in [1/2, 1)
  const int e = amax > 0.f ? x - 3 + (m > 0.875f ? 1 : 0) : kExpMin;
  return min(max(e, kExpMin), kExpMax);
}

// Eight elements to codes, element i in bits 4 i, and the exponent of the 32 that this lane and its three neighbours have
template <bool BF16>
__device__ __forceinline__ u32 quantise(const uint4& raw, int& e) {
  float f[8], top = 0.f;
  cvt8<BF16>(raw, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!(f[i] == f[i])) f[i] = 0.f;           // a NaN becomes 0
    const float m = fabsf(f[i]);
    top = fmaxf(top, m < INFINITY ? m : 0.f);
  }
  top = fmaxf(top, dpp_mov<0xB1>(top));        // quad_perm 1 0 3 2
  top = fmaxf(top, dpp_mov<0x4E>(top));        // quad_perm 2 3 0 1
  e = exp_for(top);
  const float scale = two_to(e);
  u32 w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
  return w;
}

// One workgroup for a run and a head, a tile at a time.  A tile is put together in LDS, on top of what it held where some of that
// stays, and stored whole, 16 bytes a lane.
template <bool BF16>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  __shared__ __align__(16) unsigned char tile[kTileBytes];
  const int tid = threadIdx.x, lane = tid % kWave, t = tid >> 4, j = tid & 15;
  const int h = blockIdx.y;
  const int4 run = a.runs[blockIdx.x];
  const int block = run.x, row0 = run.y, off = run.z, n = run.w;
  if ((unsigned)block >= (unsigned)a.NB || off < 0 || n < 1 || n > a.P - off || row0 < 0 || n > a.T - row0) return;
  const int end = off + n;
  const bool begins = off == 0;
  unsigned char* page = a.pages + ((size_t)block * a.H + h) * (a.P / kTile) * kTileBytes;
  const uint16_t* kp = a.k + ((long long)row0 - off) * a.k_stride + h * kHeadDim + j * 8;
  const uint16_t* vp = a.v + ((long long)row0 - off) * a.v_stride + h * kHeadDim + j * 8;
  const int last = begins ? a.P / kTile : (end + kTile - 1) / kTile;
  uint4 rk = make_uint4(0, 0, 0, 0), rv = rk, old = rk;
  auto stays = [&](int i) { return !begins && (i * kTile < off || (i + 1) * kTile > end); };
  auto fetch = [&](int i) {
    const int tok = i * kTile + t;
    if (tok >= off && tok < end) {
      rk = *reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride);
      rv = *reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride);
    }
    if (stays(i) && tid < kTileBytes / 16) old = *reinterpret_cast<const uint4*>(page + (size_t)i * kTileBytes + tid * 16);
  };
  fetch(off / kTile);
  for (int i = off / kTile; i < last; ++i) {
    const int tok = i * kTile + t;
    const bool fresh = tok >= off && tok < end, keeps = stays(i);
    if (keeps) {
      if (tid < kTileBytes / 16) *reinterpret_cast<uint4*>(tile + tid * 16) = old;
      __syncthreads();
    }
    int ek, ev;
    u32 ck = quantise<BF16>(rk, ek), cv = quantise<BF16>(rv, ev);
    if (!fresh) { ck = cv = 0; ek = ev = kExpMin; }
    if (i + 1 < last) fetch(i + 1);
    if (fresh || !keeps) {
      *reinterpret_cast<u32*>(tile + t * 64 + j * 4) = ck;
      if ((j & 3) == 0) {
        tile[kKeyScales + (j >> 2) * 16 + (t & 3) * 4 + (t >> 2)] = (unsigned char)(ek + kBias);
        tile[kValueScales + (j >> 2) * 16 + t] = (unsigned char)(ev + kBias);
      }
    }
    // the codes of four tokens, which are lanes of one wave, two of the eight elements a lane
    const u32 c0 = __shfl(cv, j, kWave), c1 = __shfl(cv, j + 16, kWave), c2 = __shfl(cv, j + 32, kWave), c3 = __shfl(cv, j + 48, kWave);
    const int first = i * kTile + (t & ~3);    // position of the first of the four
    u32 mask = 0xffff;
    if (keeps) {
      mask = 0;
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (first + y >= off && first + y < end) mask |= 15u << (4 * y);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int x = (lane >> 4) * 2 + y, d = j * 8 + x, s = 4 * x;
      const u32 w = (c0 >> s & 15) | (c1 >> s & 15) << 4 | (c2 >> s & 15) << 8 | (c3 >> s & 15) << 12;
      uint16_t* to = reinterpret_cast<uint16_t*>(tile + kValues + (d >> 5) * 256 + (d & 15) * 16 + ((d >> 4) & 1) * 8) + (t >> 2);
      *to = (uint16_t)(keeps ? (*to & ~mask) | (w & mask) : w);
    }
    __syncthreads();
    if (tid < kTileBytes / 16) *reinterpret_cast<uint4*>(page + (size_t)i * kTileBytes + tid * 16) = *reinterpret_cast<const uint4*>(tile + tid * 16);
    __syncthreads();
  }
}

// ---- reading back

constexpr int kReadThreads = 256, kReadRows = kReadThreads / 8;          // 8 lanes have a row, 16 elements each

struct ReadArgs {
  uint16_t *k, *v;
  long long k_stride, v_stride;
  const int32_t *table, *row_seq, *row_pos;
  const unsigned char* pages;
  int B, NP, T, H, P, NB;
};

// Two codes of a byte to two elements; f16 has no 6 * 2^14: the largest number it has stands for more
template <bool BF16>
__device__ __forceinline__ u32 widen2(u32 byte, float scale) {
  const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, scale, 0);
  if (BF16) return pack2<true>(x[0], x[1]);
  return pack2<false>(fminf(fmaxf(x[0], -65504.f), 65504.f), fminf(fmaxf(x[1], -65504.f), 65504.f));
}

template <bool BF16>
__global__ __launch_bounds__(kReadThreads) void read_kernel(ReadArgs a) {
  const int tid = threadIdx.x, j = tid & 7, h = blockIdx.y;
  const int row = blockIdx.x * kReadRows + (tid >> 3);
  if (row >= a.T) return;
  const int seq = a.row_seq[row], pos = a.row_pos[row];
  if ((unsigned)seq >= (unsigned)a.B || pos < 0 || pos >= a.NP * a.P) return;
  const int block = a.table[(size_t)seq * a.NP + pos / a.P];
  if ((unsigned)block >= (unsigned)a.NB) return;
  const int t = pos % kTile;
  const unsigned char* tile = a.pages + (((size_t)block * a.H + h) * (a.P / kTile) + pos % a.P / kTile) * kTileBytes;
  const uint2 kc = *reinterpret_cast<const uint2*>(tile + t * 64 + j * 8);
  const unsigned char* vp = tile + kValues + (j >> 1) * 256 + (j & 1) * 8 + (t >> 1);
  u32 vb[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) vb[i] = vp[i * 16];
  const float ks = two_to(tile[kKeyScales + (j >> 1) * 16 + (t & 3) * 4 + (t >> 2)] - kBias);
  const float vs = two_to(tile[kValueScales + (j >> 1) * 16 + t] - kBias);
  u32 w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = widen2<BF16>(((i < 4 ? kc.x : kc.y) >> (8 * (i & 3))) & 255, ks);
  uint4* to = reinterpret_cast<uint4*>(a.k + (long long)row * a.k_stride + h * kHeadDim + j * 16);
  to[0] = make_uint4(w[0], w[1], w[2], w[3]);
  to[1] = make_uint4(w[4], w[5], w[6], w[7]);
  const int s = (t & 1) * 4;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = widen2<BF16>((vb[2 * i] >> s & 15) | (vb[2 * i + 1] >> s & 15) << 4, vs);
  to = reinterpret_cast<uint4*>(a.v + (long long)row * a.v_stride + h * kHeadDim + j * 16);
  to[0] = make_uint4(w[0], w[1], w[2], w[3]);
  to[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

}  // namespace q4
}  // namespace kvd

extern "C" int kvd_q4_append(const kvd_q4_cache* c, const kvd_q8_rows* r, const void* k_new, int64_t k_stride,
                             const void* v_new, int64_t v_stride, void* stream) {
  using namespace kvd::q4;
  if (int e = check_cache(c, r)) return e;
  if (!aligned(c->pages, 128) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(r->runs, 16)) return KVD_ERR_ARG;
  if (!stride_ok(k_stride, c->n_kv_heads) || !stride_ok(v_stride, c->n_kv_heads)) return KVD_ERR_SHAPE;
  AppendArgs a;
  a.k = static_cast<const uint16_t*>(k_new); a.v = static_cast<const uint16_t*>(v_new);
  a.k_stride = k_stride; a.v_stride = v_stride;
  a.runs = reinterpret_cast<const int4*>(r->runs);
  a.pages = static_cast<unsigned char*>(c->pages);
  a.H = c->n_kv_heads; a.P = c->page_size; a.NB = c->n_blocks; a.T = r->n_rows;
  const dim3 grid(r->max_runs, c->n_kv_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->kv_dtype == KVD_BF16) hipLaunchKernelGGL(append_kernel<true>, grid, dim3(kAppendThreads), 0, s, a);
  else hipLaunchKernelGGL(append_kernel<false>, grid, dim3(kAppendThreads), 0, s, a);
  return launched();
}

extern "C" int kvd_q4_read(const kvd_q4_cache* c, const kvd_q8_rows* r, void* k, int64_t k_stride, void* v, int64_t v_stride,
                           void* stream) {
  using namespace kvd::q4;
  if (int e = check_cache(c, r)) return e;
  if (!aligned(c->pages, 128) || !aligned(k, 16) || !aligned(v, 16)) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->row_seq, 4) || !aligned(r->row_pos, 4)) return KVD_ERR_ARG;
  if (!stride_ok(k_stride, c->n_kv_heads) || !stride_ok(v_stride, c->n_kv_heads)) return KVD_ERR_SHAPE;
  ReadArgs a;
  a.k = static_cast<uint16_t*>(k); a.v = static_cast<uint16_t*>(v);
  a.k_stride = k_stride; a.v_stride = v_stride;
  a.table = r->page_table; a.row_seq = r->row_seq; a.row_pos = r->row_pos;
  a.pages = static_cast<const unsigned char*>(c->pages);
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.H = c->n_kv_heads; a.P = c->page_size; a.NB = c->n_blocks;
  const dim3 grid((a.T + kReadRows - 1) / kReadRows, a.H);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->kv_dtype == KVD_BF16) hipLaunchKernelGGL(read_kernel<true>, grid, dim3(kReadThreads), 0, s, a);
  else hipLaunchKernelGGL(read_kernel<false>, grid, dim3(kReadThreads), 0, s, a);
  return launched();
}
