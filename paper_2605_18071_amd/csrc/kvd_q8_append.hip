// Quantises a step's new keys and values into their pages: one workgroup for the new tokens of one page (a run) and one
// head.  The largest magnitude gives the scale 2^e, the elements times 2^-e go to e4m3 by the hardware's conversion,
// which rounds to nearest even; products with powers of two are exact, so that there is no rounding but that one.  Codes are
// put together in LDS, tile by tile, so that the pool is written 16 bytes a lane.  Bound by the memory: 4 bytes read and
// 2 written for an element of a key and its value's.
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kAppendThreads = 256;            // 16 tokens x 16 lanes of 8 elements: a tile's keys, then its values

struct AppendArgs {
  const uint16_t *k, *v;
  long long k_stride, v_stride;
  const int4* runs;
  unsigned char* pages;
  int8_t *exps, *means;
  float* mean_scales;
  int H, P, NB, T;
};

// The least e >= kExpMin with amax <= 448 * 2^e; amax finite.  (448 = 1.75 * 2^8)
__device__ __forceinline__ int exp_for(float amax) {
  int x;
  const float m = frexpf(amax, &x);            // m in [1/2, 1)
  if (!(amax > 0.f)) return kExpMin;
  const int e = x - 9 + (m > 0.875f ? 1 : 0);
  return e > kExpMin ? e : kExpMin;
}
// Magnitude of a finite element, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// An element times 2^-e into the range of the codes
__device__ __forceinline__ float in_range(float x, float scale) {
  const float y = fminf(fmaxf(x * scale, -448.f), 448.f);
  return x == x ? y : 0.f;
}
__device__ __forceinline__ u32 code4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (u32)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void values4(u32 w, float (&f)[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
// Codes of a scale 2^e to a scale that is 2^-shift as fine
__device__ __forceinline__ u32 rescale4(u32 w, float shift) {
  float f[4];
  values4(w, f);
  return code4(f[0] * shift, f[1] * shift, f[2] * shift, f[3] * shift);
}

template <bool BF16>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  __shared__ __align__(16) unsigned char tile[kTileBytes];
  __shared__ float red[2][kAppendThreads / kWave];
  __shared__ int sums[kAppendThreads / kWave][kHeadDim];
  __shared__ int red_max[2];
  const int tid = threadIdx.x, w = tid / kWave, t = tid >> 4, d0 = (tid & 15) * 8;
  const int h = blockIdx.y;
  const int4 run = a.runs[blockIdx.x];
  const int block = run.x, row0 = run.y, off = run.z, n = run.w;
  if ((unsigned)block >= (unsigned)a.NB || off < 0 || n < 1 || n > a.P - off || row0 < 0 || n > a.T - row0) return;
  const int end = off + n;
  const size_t unit = (size_t)block * a.H + h;
  unsigned char* page = a.pages + unit * (a.P / kTile) * kTileBytes;
  const uint16_t* kp = a.k + ((long long)row0 - off) * a.k_stride + h * kHeadDim + d0;
  const uint16_t* vp = a.v + ((long long)row0 - off) * a.v_stride + h * kHeadDim + d0;

  float mk = 0.f, mv = 0.f;
  for (int tok = off / kTile * kTile + t; tok < end; tok += kTile)
    if (tok >= off) {
      float f[8], g[8];
      cvt8<BF16>(*reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride), f);
      cvt8<BF16>(*reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride), g);
#pragma unroll
      for (int i = 0; i < 8; ++i) { mk = fmaxf(mk, finite_abs(f[i])); mv = fmaxf(mv, finite_abs(g[i])); }
    }
  mk = wave_allreduce_max(mk);
  mv = wave_allreduce_max(mv);
  if (tid % kWave == 0) { red[0][w] = mk; red[1][w] = mv; }
  const bool begins = off == 0;
  int was_k = 0, was_v = 0;
  if (!begins) { was_k = a.exps[unit * 2]; was_v = a.exps[unit * 2 + 1]; }
  __syncthreads();                             // (every thread has the old exponents before they are replaced)
#pragma unroll
  for (int i = 0; i < kAppendThreads / kWave; ++i) { mk = fmaxf(mk, red[0][i]); mv = fmaxf(mv, red[1][i]); }
  int ek = exp_for(mk), ev = exp_for(mv);
  if (!begins) { ek = max(ek, was_k); ev = max(ev, was_v); }
  const float sk = two_to(-ek), sv = two_to(-ev);
  const bool regrade_k = !begins && ek != was_k, regrade_v = !begins && ev != was_v;
  const float shift_k = two_to(max(was_k - ek, -126)), shift_v = two_to(max(was_v - ev, -126));

  int sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int last = begins ? a.P / kTile : (end + kTile - 1) / kTile;
  for (int ti = 0; ti < last; ++ti) {
    unsigned char* at = page + (size_t)ti * kTileBytes;
    const int tok = ti * kTile + t;
    const bool held = !begins && (ti * kTile < off || ti == last - 1);     // the tile has codes that stay
    __syncthreads();
    if (held) *reinterpret_cast<uint4*>(tile + tid * 16) = *reinterpret_cast<const uint4*>(at + tid * 16);
    __syncthreads();
    u32* kc = reinterpret_cast<u32*>(tile + key_at(t, d0));
    unsigned char* vc = tile + kHalfTile;
    if (tok >= off && tok < end) {
      float f[8], g[8];
      cvt8<BF16>(*reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride), f);
      cvt8<BF16>(*reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride), g);
#pragma unroll
      for (int i = 0; i < 8; ++i) { f[i] = in_range(f[i], sk); g[i] = in_range(g[i], sv); }
      kc[0] = code4(f[0], f[1], f[2], f[3]);
      kc[1] = code4(f[4], f[5], f[6], f[7]);
      const u32 v0 = code4(g[0], g[1], g[2], g[3]), v1 = code4(g[4], g[5], g[6], g[7]);
#pragma unroll
      for (int i = 0; i < 8; ++i) vc[value_at(t, d0 + i)] = (unsigned char)((i < 4 ? v0 : v1) >> ((i & 3) * 8));
    } else if (tok < off) {
      if (regrade_k) { kc[0] = rescale4(kc[0], shift_k); kc[1] = rescale4(kc[1], shift_k); }
      if (regrade_v)
        for (int i = 0; i < 8; ++i) {
          unsigned char* c = vc + value_at(t, d0 + i);
          *c = (unsigned char)rescale4(*c, shift_v);
        }
    } else if (begins) {
      kc[0] = kc[1] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) vc[value_at(t, d0 + i)] = 0;
    }
    if (tok < end) {
      float f[4], g[4];
      values4(kc[0], f);
      values4(kc[1], g);
#pragma unroll
      for (int i = 0; i < 4; ++i) { sum[i] += (int)(f[i] * 512.f); sum[4 + i] += (int)(g[i] * 512.f); }
    }
    __syncthreads();
    *reinterpret_cast<uint4*>(at + tid * 16) = *reinterpret_cast<const uint4*>(tile + tid * 16);
  }
  if (tid == 0) {
    a.exps[unit * 2] = (int8_t)ek;
    a.exps[unit * 2 + 1] = (int8_t)ev;
  }
  // the index entry: sums over the tokens, by lanes 16 apart, then by waves
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sum[i] += __shfl_xor(sum[i], 16, kWave);
    sum[i] += __shfl_xor(sum[i], 32, kWave);
  }
  if (tid % kWave < 16)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[w][d0 + i] = sum[i];
  __syncthreads();
  if (tid < kHeadDim) {
    int s = 0;
#pragma unroll
    for (int i = 0; i < kAppendThreads / kWave; ++i) s += sums[i][tid];
    int m = abs(s);
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) m = max(m, __shfl_xor(m, x, kWave));
    if (tid % kWave == 0) red_max[w] = m;
    sum[0] = s;
  }
  __syncthreads();
  if (tid < kHeadDim) {
    const int m = max(red_max[0], red_max[1]);       // below 2^27
    int sh = 0;
    while (m > (127 << sh)) ++sh;
    // (the sum has up to 27 bits: halves are kept apart by fp64)
    a.means[unit * kHeadDim + tid] = (int8_t)rint((double)sum[0] * (double)two_to(-sh));
    if (tid == 0) a.mean_scales[unit] = (float)(ldexp(1.0, sh - 9 + ek) / (double)end);
  }
}

}  // namespace q8
}  // namespace kvd

extern "C" int kvd_q8_append(const kvd_q8_cache* c, const kvd_q8_rows* r, const void* k_new, int64_t k_stride,
                             const void* v_new, int64_t v_stride, void* stream) {
  using namespace kvd::q8;
  if (int e = check_cache(c, r)) return e;
  if (!aligned(c->pages, 16) || !aligned(c->exps, 2) || !aligned(c->means, 16) || !aligned(c->mean_scales, 4)) return KVD_ERR_ARG;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(r->runs, 16)) return KVD_ERR_ARG;
  if (!stride_ok(k_stride, c->n_kv_heads) || !stride_ok(v_stride, c->n_kv_heads)) return KVD_ERR_SHAPE;
  AppendArgs a;
  a.k = static_cast<const uint16_t*>(k_new); a.v = static_cast<const uint16_t*>(v_new);
  a.k_stride = k_stride; a.v_stride = v_stride;
  a.runs = reinterpret_cast<const int4*>(r->runs);
  a.pages = static_cast<unsigned char*>(c->pages); a.exps = c->exps; a.means = c->means; a.mean_scales = c->mean_scales;
  a.H = c->n_kv_heads; a.P = c->page_size; a.NB = c->n_blocks; a.T = r->n_rows;
  const dim3 grid(r->max_runs, c->n_kv_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->kv_dtype == KVD_BF16) hipLaunchKernelGGL(append_kernel<true>, grid, dim3(kAppendThreads), 0, s, a);
  else hipLaunchKernelGGL(append_kernel<false>, grid, dim3(kAppendThreads), 0, s, a);
  return launched();
}
