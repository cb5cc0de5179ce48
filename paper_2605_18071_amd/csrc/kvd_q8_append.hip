// Quantises a step's new keys and values into their pages: one workgroup for the new tokens of one page (a run) and one
// head.  The largest magnitude gives the scale 2^e, the elements times 2^-e go to e4m3 by the hardware's conversion,
// which rounds to nearest even; products with powers of two are exact, so that there is no rounding but that one.  Codes are
// put together in LDS, so that the pool is written 16 bytes a lane.  Bound by the memory: 4 bytes read and
// 2 written for an element of a key and its value's (32768 tokens of 8 heads 44 us, 4.6 TB/s, and 50 where the card has run for
// long; a token for each of 64 requests 5.2).
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

// MT tiles at a time; a page of no more is read once and kept in registers (WHOLE), of a larger one the new tokens are read
// again, out of the cache.  What the page holds before the run is asked for together with the run's tokens: a step that adds a token
// to each page is a chain of trips to memory, and nothing else.
template <bool BF16, int MT, bool WHOLE>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  constexpr int NW = kAppendThreads / kWave;
  __shared__ __align__(16) unsigned char tile[MT][kTileBytes];
  __shared__ float red[2][NW];
  __shared__ int sums[NW][kHeadDim];
  const int tid = threadIdx.x, w = tid / kWave, lane = tid % kWave, t = tid >> 4, d0 = (tid & 15) * 8;
  const int h = blockIdx.y;
  const int4 run = a.runs[blockIdx.x];
  const int block = run.x, row0 = run.y, off = run.z, n = run.w;
  if ((unsigned)block >= (unsigned)a.NB || off < 0 || n < 1 || n > a.P - off || row0 < 0 || n > a.T - row0) return;
  const int end = off + n;
  const bool begins = off == 0;
  const size_t unit = (size_t)block * a.H + h;
  unsigned char* page = a.pages + unit * (a.P / kTile) * kTileBytes;
  const uint16_t* kp = a.k + ((long long)row0 - off) * a.k_stride + h * kHeadDim + d0;
  const uint16_t* vp = a.v + ((long long)row0 - off) * a.v_stride + h * kHeadDim + d0;
  const int last = begins ? a.P / kTile : (end + kTile - 1) / kTile;   // tiles that are written, from the first
  // tiles with codes that stay: those before the run's first token and the one of its last
  auto held = [&](int ti) { return !begins && (ti * kTile < off || ti == last - 1); };
  auto is_new = [&](int tok) { return tok >= off && tok < end; };

  uint4 rk[MT], rv[MT], old[MT];
  float mk = 0.f, mv = 0.f;
  auto largest = [&](const uint4& x, const uint4& y) {
    float f[8], g[8];
    cvt8<BF16>(x, f);
    cvt8<BF16>(y, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) { mk = fmaxf(mk, finite_abs(f[i])); mv = fmaxf(mv, finite_abs(g[i])); }
  };
  int was_k = 0, was_v = 0;
  if (!begins) { was_k = a.exps[unit * 2]; was_v = a.exps[unit * 2 + 1]; }
  if (WHOLE) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int tok = i * kTile + t;
      if (is_new(tok)) {
        rk[i] = *reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride);
        rv[i] = *reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride);
      }
      if (i < last && held(i)) old[i] = *reinterpret_cast<const uint4*>(page + i * kTileBytes + tid * 16);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
      if (is_new(i * kTile + t)) largest(rk[i], rv[i]);
  } else {
    for (int tok = off / kTile * kTile + t; tok < end; tok += kTile)
      if (tok >= off)
        largest(*reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride), *reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride));
  }
  mk = wave_allreduce_max(mk);
  mv = wave_allreduce_max(mv);
  if (lane == 0) { red[0][w] = mk; red[1][w] = mv; }
  __syncthreads();                             // (every thread has the old exponents before they are replaced)
#pragma unroll
  for (int i = 0; i < NW; ++i) { mk = fmaxf(mk, red[0][i]); mv = fmaxf(mv, red[1][i]); }
  int ek = exp_for(mk), ev = exp_for(mv);
  if (!begins) { ek = max(ek, was_k); ev = max(ev, was_v); }
  const float sk = two_to(-ek), sv = two_to(-ev);
  const bool regrade_k = !begins && ek != was_k, regrade_v = !begins && ev != was_v;
  const float shift_k = two_to(max(was_k - ek, -126)), shift_v = two_to(max(was_v - ev, -126));
  if (tid == 0) {
    a.exps[unit * 2] = (int8_t)ek;
    a.exps[unit * 2 + 1] = (int8_t)ev;
  }

  int sum0 = 0, sum1 = 0;                      // of elements 2 lane and 2 lane + 1 over the tiles that are this wave's
  for (int c0 = 0; c0 < (WHOLE ? 1 : last); c0 += MT) {
    if (!WHOLE) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int tok = (c0 + i) * kTile + t;
        if (is_new(tok)) {
          rk[i] = *reinterpret_cast<const uint4*>(kp + (long long)tok * a.k_stride);
          rv[i] = *reinterpret_cast<const uint4*>(vp + (long long)tok * a.v_stride);
        }
        if (c0 + i < last && held(c0 + i)) old[i] = *reinterpret_cast<const uint4*>(page + (size_t)(c0 + i) * kTileBytes + tid * 16);
      }
      __syncthreads();                         // (the tiles before these have been stored)
    }
    if (!begins) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
        if (c0 + i < last && held(c0 + i)) *reinterpret_cast<uint4*>(tile[i] + tid * 16) = old[i];
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int tok = (c0 + i) * kTile + t;
      if (c0 + i >= last) break;
      u32* kc = reinterpret_cast<u32*>(tile[i] + key_at(t, d0));
      unsigned char* vc = tile[i] + kHalfTile + value_at(t, d0);         // (of element d0 + y: 16 bytes on)
      if (is_new(tok)) {
        float f[8], g[8];
        cvt8<BF16>(rk[i], f);
        cvt8<BF16>(rv[i], g);
#pragma unroll
        for (int y = 0; y < 8; ++y) { f[y] = in_range(f[y], sk); g[y] = in_range(g[y], sv); }
        kc[0] = code4(f[0], f[1], f[2], f[3]);
        kc[1] = code4(f[4], f[5], f[6], f[7]);
        const u32 v0 = code4(g[0], g[1], g[2], g[3]), v1 = code4(g[4], g[5], g[6], g[7]);
#pragma unroll
        for (int y = 0; y < 8; ++y) vc[y * 16] = (unsigned char)((y < 4 ? v0 : v1) >> ((y & 3) * 8));
      } else if (tok < off) {
        if (regrade_k) { kc[0] = rescale4(kc[0], shift_k); kc[1] = rescale4(kc[1], shift_k); }
        if (regrade_v)
          for (int y = 0; y < 8; ++y) vc[y * 16] = (unsigned char)rescale4(vc[y * 16], shift_v);
      } else if (begins) {
        kc[0] = kc[1] = 0;
#pragma unroll
        for (int y = 0; y < 8; ++y) vc[y * 16] = 0;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
      if (c0 + i < last)
        *reinterpret_cast<uint4*>(page + (size_t)(c0 + i) * kTileBytes + tid * 16) = *reinterpret_cast<const uint4*>(tile[i] + tid * 16);
    // sums of the keys' codes: a wave a tile, below 2^13 in steps of 2^-9, which fp32 holds exactly
#pragma unroll
    for (int i = 0; i < MT; ++i)
      if (i % NW == w && c0 + i < last) {
        const int count = min(max(end - (c0 + i) * kTile, 0), kTile);
        const unsigned char* at = tile[i] + key_at(0, 2 * lane);
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int y = 0; y < kTile; ++y) {
          const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(*reinterpret_cast<const uint16_t*>(at + y * 16), false);
          if (y < count) { s0 += x.x; s1 += x.y; }
        }
        sum0 += (int)(s0 * 512.f);
        sum1 += (int)(s1 * 512.f);
      }
  }
  if (MT > 1) {
    sums[w][2 * lane] = sum0;
    sums[w][2 * lane + 1] = sum1;
    __syncthreads();
    sum0 = sum1 = 0;
#pragma unroll
    for (int i = 0; i < (MT < NW ? MT : NW); ++i) { sum0 += sums[i][2 * lane]; sum1 += sums[i][2 * lane + 1]; }
  }
  if (w == 0) {                                // the index entry
    int m = max(abs(sum0), abs(sum1));         // below 2^27
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) m = max(m, __shfl_xor(m, x, kWave));
    int sh = 0;
    while (m > (127 << sh)) ++sh;
    // (the sum has up to 27 bits: halves are kept apart by fp64)
    const double scale = (double)two_to(-sh);
    const int m0 = (int)rint((double)sum0 * scale), m1 = (int)rint((double)sum1 * scale);
    *reinterpret_cast<uint16_t*>(a.means + unit * kHeadDim + 2 * lane) = (uint16_t)((m0 & 0xff) | (m1 & 0xff) << 8);
    if (lane == 0) a.mean_scales[unit] = (float)(ldexp(1.0, sh - 9 + ek) / (double)end);
  }
}

template <bool BF16>
static void launch_append(const AppendArgs& a, dim3 grid, hipStream_t s) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kAppendThreads), 0, s, a); };
  const int tiles = a.P / kTile;
  if (tiles == 1) go(append_kernel<BF16, 1, true>);
  else if (tiles == 2) go(append_kernel<BF16, 2, true>);
  else if (tiles <= 4) go(append_kernel<BF16, 4, true>);
  else go(append_kernel<BF16, 4, false>);
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
  if (c->kv_dtype == KVD_BF16) launch_append<true>(a, grid, s);
  else launch_append<false>(a, grid, s);
  return launched();
}
