// Norm and rotation of a step's query and key heads in one pass: y = x / sqrt(mean x^2 + eps) * w, then pairs of elements turned
// by their position's angle, rounded once.  Angles are turns, position * frequency / 2 pi in twice fp64, of which the fraction is kept.
// Bound by the memory, 2 bytes an element read and 2 written:
// 32768 rows of 32 + 8 heads 121 us (5.5 TB/s; a copy of as many bytes takes 130), a step of 64 rows 3.8 (the launch and a trip to memory
// and back).  Sines are the work of one thread for each pair and row, and shared by the row's heads through LDS; 16 lanes have
// kAhead heads on their way (154 us with one).
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kRotThreads = 256;
constexpr int kMaxPairs = kHeadDim / 2;
constexpr int kMaxRotRows = 1 << 24;
constexpr int kMaxRotHeads = 65536;
constexpr int kAhead = 4;                      // heads on their way to 16 lanes

struct RotateArgs {
  const uint16_t *q, *k, *q_weight, *k_weight;
  uint16_t *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride, pos_stride;
  const int32_t* pos;
  const float* inv_freq;
  int T, Hq, Hk, pairs, axis_end[4];           // axis_end: first pair behind the axis
  float eps;
};

// What pos * freq / 2 pi turns have beyond whole ones, off by 2^-25 of a turn at most up to 2^50 turns.  The product has 55 bits, so p and
// p_rest are all of it, and kPerRadian and kRest are 106 bits of 1 / 2 pi; with 53 of each 5e8 turns were off by 1.5 * 2^-24.
__device__ __forceinline__ float fraction(int pos, float freq) {
  constexpr double kPerRadian = 0.15915494309189535, kRest = -9.839338337591243e-18;
  const double x = (double)pos, f = (double)freq, p = x * f, p_rest = __builtin_fma(x, f, -p);
  return (float)(__builtin_fma(p, kPerRadian, -rint(p * kPerRadian)) + (p * kRest + p_rest * kPerRadian));
}

// Cosine and sine of r turns, r in -1/2..1/2: quarter turns taken off, then their series, off by 2^-25 where they end
__device__ __forceinline__ float2 cos_sin(float r) {
  const float quarters = rintf(4.f * r), x = 6.28318530717958648f * (r - 0.25f * quarters), x2 = x * x;     // |x| <= pi / 4
  const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
  const float c = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
  const int q = (int)quarters & 3;
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -a : a, q & 2 ? -b : b);
}

// NR rows a workgroup; 16 lanes have a head, 8 elements each.  NEAR: a pair's elements are neighbours, else `pairs` apart.
template <bool BF16, bool NEAR, int NR>
__global__ __launch_bounds__(kRotThreads) void norm_rotate_kernel(RotateArgs a) {
  constexpr int kGroups = kRotThreads / 16;    // heads at a time
  __shared__ float2 turn[NR][kMaxPairs];
  const int tid = threadIdx.x, j = tid & 15, group = tid >> 4;
  const long long row0 = (long long)blockIdx.x * NR;
  const long long row = row0 + group % NR;
  const int heads = a.Hq + a.Hk, per = kGroups / NR * gridDim.y;
  int head = blockIdx.y * (kGroups / NR) + group / NR;
  // everything is asked for at the beginning, whether the row has a token or not
  const int place = row < a.T ? a.pos[row] : -1;
  auto at = [&](int h) {
    return h < a.Hq ? a.q + row * a.q_stride + (long long)h * kHeadDim + j * 8
                    : a.k + row * a.k_stride + (long long)(h - a.Hq) * kHeadDim + j * 8;
  };
  uint4 x[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    x[i] = make_uint4(0, 0, 0, 0);
    if (row < a.T && head + i * per < heads) x[i] = *reinterpret_cast<const uint4*>(at(head + i * per));
  }
  const int half = a.pairs / 8;                // lanes of the first elements of pairs that lie apart
  const bool turned = j < 2 * half, second = !NEAR && j >= half;
  const int lane = tid % kWave, partner = (lane & ~15) + (turned ? (second ? j - half : j + half) : j);
  // weights: of the lane's elements and of its partner's, of both kinds of heads
  uint4 wq = make_uint4(0, 0, 0, 0), wk = wq, vq = wq, vk = wq;
  if (a.q_weight) {
    wq = *reinterpret_cast<const uint4*>(a.q_weight + j * 8);
    vq = *reinterpret_cast<const uint4*>(a.q_weight + (partner & 15) * 8);
  }
  if (a.k_weight) {
    wk = *reinterpret_cast<const uint4*>(a.k_weight + j * 8);
    vk = *reinterpret_cast<const uint4*>(a.k_weight + (partner & 15) * 8);
  }
  for (int i = tid; i < NR * kMaxPairs; i += kRotThreads) {
    const int r = i / kMaxPairs, p = i % kMaxPairs;
    if (p < a.pairs && row0 + r < a.T) {
      const int axis = (p >= a.axis_end[0]) + (p >= a.axis_end[1]) + (p >= a.axis_end[2]);
      turn[r][p] = cos_sin(fraction(a.pos[axis * a.pos_stride + row0 + r], a.inv_freq[p]));
    }
  }
  __syncthreads();
  // the lane's cosines and sines: of its four pairs, or of the eight that its elements are one half of
  float2 t[NEAR ? 4 : 8];
  if (turned)
#pragma unroll
    for (int i = 0; i < (NEAR ? 4 : 8); ++i) t[i] = turn[group % NR][NEAR ? j * 4 + i : (second ? j - half : j) * 8 + i];
  if (place < 0) return;                       // (whole groups of 16 lanes)
  for (; head < heads; head += kAhead * per) {
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      const int hd = head + y * per;
      if (hd >= heads) break;
      const bool is_q = hd < a.Hq, norm = (is_q ? a.q_weight : a.k_weight) != nullptr;
      const uint4 raw = x[y];
      if (hd + kAhead * per < heads) x[y] = *reinterpret_cast<const uint4*>(at(hd + kAhead * per));
      float f[8], g[8];
      cvt8<BF16>(raw, f);
      if (!NEAR) {
        const uint4 other = make_uint4(__shfl(raw.x, partner, kWave), __shfl(raw.y, partner, kWave), __shfl(raw.z, partner, kWave),
                                       __shfl(raw.w, partner, kWave));
        cvt8<BF16>(other, g);
      }
      if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += f[i] * f[i];
        const float inv = rsqrtf(row16_allreduce_sum(sum) * (1.f / kHeadDim) + a.eps);
        const uint4 mine = is_q ? wq : wk, theirs = is_q ? vq : vk;
        float w[8];
        cvt8<BF16>(mine, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= inv * w[i];
        if (!NEAR) {
          cvt8<BF16>(theirs, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) g[i] *= inv * w[i];
        }
      }
      if (turned) {
        if constexpr (NEAR) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float u = f[2 * i], v = f[2 * i + 1];
            f[2 * i] = u * t[i].x - v * t[i].y;
            f[2 * i + 1] = u * t[i].y + v * t[i].x;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = second ? g[i] * t[i].y + f[i] * t[i].x : f[i] * t[i].x - g[i] * t[i].y;
        }
      }
      uint16_t* to = is_q ? a.q_out + row * a.q_out_stride + (long long)hd * kHeadDim + j * 8
                          : a.k_out + row * a.k_out_stride + (long long)(hd - a.Hq) * kHeadDim + j * 8;
      *reinterpret_cast<uint4*>(to) = make_uint4(pack2<BF16>(f[0], f[1]), pack2<BF16>(f[2], f[3]), pack2<BF16>(f[4], f[5]), pack2<BF16>(f[6], f[7]));
    }
  }
}

template <bool BF16, bool NEAR>
static void launch_rotate(const RotateArgs& a, hipStream_t s) {
  // Few rows are spread over the CUs, a row each, the fewest with their heads in two workgroups; many share the workgroups' beginning.  us
  // with a row in two workgroups, in one, and four rows in one, 32 + 8 heads: 256 rows 4.1, 4.5, 7.2; 1000 7.8, 7.1, 8.6; 2000 12.9, 11.8,
  // 12.0; 10000 60, 48, 45.
  if (a.T >= 2048) hipLaunchKernelGGL((norm_rotate_kernel<BF16, NEAR, 4>), dim3((a.T + 3) / 4), dim3(kRotThreads), 0, s, a);
  else hipLaunchKernelGGL((norm_rotate_kernel<BF16, NEAR, 1>), dim3(a.T, a.T <= 256 && a.Hq + a.Hk > 16 ? 2 : 1), dim3(kRotThreads), 0, s, a);
}

}  // namespace q8
}  // namespace kvd

extern "C" int kvd_norm_rotate(const kvd_rotary* c, const int32_t* pos, int64_t pos_stride, int32_t n_rows, const void* q,
                               int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out,
                               int64_t k_out_stride, void* stream) {
  using namespace kvd::q8;
  if (!c) return KVD_ERR_ARG;
  if (c->kv_dtype != KVD_F16 && c->kv_dtype != KVD_BF16) return KVD_ERR_DTYPE;
  if (c->head_dim != kvd::kHeadDim || n_rows < 1 || n_rows > kMaxRotRows) return KVD_ERR_SHAPE;
  if (c->rot_dim < 0 || c->rot_dim > kvd::kHeadDim || c->rot_dim % 16 || c->n_axes < 1 || c->n_axes > 4) return KVD_ERR_SHAPE;
  RotateArgs a = {};
  a.pairs = c->rot_dim / 2;
  int end = 0;
  for (int i = 0; i < 4; ++i) {
    if (i < c->n_axes) {
      if (c->axis_pairs[i] < 0 || c->axis_pairs[i] > a.pairs - end) return KVD_ERR_SHAPE;
      end += c->axis_pairs[i];
    }
    a.axis_end[i] = i < c->n_axes - 1 ? end : a.pairs;
  }
  if (end != a.pairs) return KVD_ERR_SHAPE;
  if (pos_stride < n_rows && c->n_axes > 1) return KVD_ERR_SHAPE;
  if (!(c->eps >= 0.f) || isinf(c->eps)) return KVD_ERR_ARG;
  if (!aligned(pos, 4) || (a.pairs > 0 && !aligned(c->inv_freq, 4)) || (!q && !k)) return KVD_ERR_ARG;
  auto tensor = [](const void* x, int64_t stride, void* out, int64_t out_stride, int heads, const void* weight) -> int {
    if (heads < 1 || heads > kMaxRotHeads || !stride_ok(stride, heads) || !stride_ok(out_stride, heads)) return KVD_ERR_SHAPE;
    if (!aligned(x, 16) || !aligned(out, 16) || (weight && !aligned(weight, 16))) return KVD_ERR_ARG;
    return x == out && stride != out_stride ? KVD_ERR_ARG : KVD_OK;
  };
  if (q) {
    if (int e = tensor(q, q_stride, q_out, q_out_stride, c->n_q_heads, c->q_weight)) return e;
    a.Hq = c->n_q_heads;
  }
  if (k) {
    if (int e = tensor(k, k_stride, k_out, k_out_stride, c->n_kv_heads, c->k_weight)) return e;
    a.Hk = c->n_kv_heads;
  }
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k);
  a.q_weight = static_cast<const uint16_t*>(c->q_weight); a.k_weight = static_cast<const uint16_t*>(c->k_weight);
  a.q_out = static_cast<uint16_t*>(q_out); a.k_out = static_cast<uint16_t*>(k_out);
  a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  a.pos_stride = pos_stride; a.pos = pos; a.inv_freq = c->inv_freq;
  a.T = n_rows; a.eps = c->eps;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->kv_dtype == KVD_BF16) {
    if (c->interleaved) launch_rotate<true, true>(a, s); else launch_rotate<true, false>(a, s);
  } else {
    if (c->interleaved) launch_rotate<false, true>(a, s); else launch_rotate<false, false>(a, s);
  }
  return launched();
}
