// Selection of pages by a score in 8 bits.  Two launches: the scores of all visible pages of every row and head, as
// products of whole numbers on the matrix cores (int8, exact, so that the result does not depend on the order), and the k best
// of a row and head by one workgroup, which holds the scores in registers.  Scoring is bound by the memory (132 bytes a page and
// head), selecting by its trips to LDS.
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 512;               // pages of a scoring workgroup
constexpr int kScoreRows = 16;                 // rows of one sequence that share its reading of the index: columns of a product
constexpr int kSelectThreads = 1024;

struct SelectArgs {
  const uint16_t* q;
  long long q_stride;
  const int32_t *table, *row_start, *row_seq, *row_pos;
  const int8_t* means;
  const float* mean_scales;
  float* scores;                               // [T][H][NP]
  int32_t* sel;
  int B, NP, T, H, G, P, NB, k, sink, recent;
};

// Pages that row r sees, 0 where it has no sequence or a position outside its table
__device__ __forceinline__ int pages_seen(const SelectArgs& a, int r, int& seq) {
  seq = a.row_seq[r];
  const int pos = a.row_pos[r];
  if ((unsigned)seq >= (unsigned)a.B || pos < 0 || pos >= a.NP * a.P) return 0;
  return pos / a.P + 1;
}

template <bool BF16>
__global__ __launch_bounds__(kScoreThreads, 4) void q8_score_kernel(SelectArgs a) {
  __shared__ __align__(16) int8_t qi[kScoreRows][kHeadDim];
  __shared__ int block_of[kScorePages];
  __shared__ int seen[kScoreRows];
  const int r0 = blockIdx.x, h = blockIdx.y, p0 = blockIdx.z * kScorePages;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  // rows r0 .. r0 + n - 1: of one sequence, for the first of which this workgroup is
  const int seq = a.row_seq[r0];
  if ((unsigned)seq >= (unsigned)a.B) return;
  // (a row is the first of its sequence, or 16, 32, ... behind it: counted back, not taken from row_start, over rows of the same sequence)
  const int back = r0 - a.row_start[seq];
  if (back < 0 || back % kScoreRows != 0) return;
  if (tid < kScoreRows) {
    int s = -1, n = 0;
    if (r0 + tid < a.T) n = pages_seen(a, r0 + tid, s);
    seen[tid] = s == seq ? n : 0;
  }
  __syncthreads();
  int most = 0;
#pragma unroll
  for (int i = 0; i < kScoreRows; ++i) most = max(most, seen[i]);
  if (p0 >= most) return;
  const int np = min(most - p0, kScorePages);
  for (int i = tid; i < np; i += kScoreThreads) block_of[i] = a.table[(size_t)seq * a.NP + p0 + i];
  // the queries in 8 bits: a wave a row, two elements a lane
  for (int i = w; i < kScoreRows; i += kScoreThreads / kWave) {
    if (seen[i] == 0) {
      *reinterpret_cast<uint16_t*>(&qi[i][lane * 2]) = 0;
      continue;
    }
    double s0 = 0.0, s1 = 0.0;
    {
      const uint16_t* q = a.q + (long long)(r0 + i) * a.q_stride + h * a.G * kHeadDim + lane * 2;
      for (int g = 0; g < a.G; ++g) {
        const u32 x = *reinterpret_cast<const u32*>(q + g * kHeadDim);
        if (BF16) { s0 += (double)as_f32(x << 16); s1 += (double)as_f32(x & 0xffff0000u); }
        else { const f16x2 v = __builtin_bit_cast(f16x2, x); s0 += (double)(float)v.x; s1 += (double)(float)v.y; }
      }
    }
    double m = fmax(fabs(s0), fabs(s1));
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) m = fmax(m, __shfl_xor(m, x, kWave));
    const double inv = 127.0 / m;
    const double a0 = s0 * inv, a1 = s1 * inv;
    qi[i][lane * 2] = fabs(a0) < 128.0 ? (int8_t)rint(a0) : 0;       // (not for NaN)
    qi[i][lane * 2 + 1] = fabs(a1) < 128.0 ? (int8_t)rint(a1) : 0;
  }
  __syncthreads();
  // 16 pages x 16 rows a product: lane l has page l % 16's (and row l % 16's) elements (l / 16) * 16 .. + 15 of each 64
  const int c = lane >> 4, n = lane & 15;
  const i32x4 q0 = *reinterpret_cast<const i32x4*>(&qi[n][c * 16]), q1 = *reinterpret_cast<const i32x4*>(&qi[n][64 + c * 16]);
  // (a wave has all its pages on their way before it takes the first)
  constexpr int N = kScorePages / (kScoreThreads / kWave * 16);
  i32x4 m0[N], m1[N];
  float scale[N];
  int good[N];
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const int t = (x * (kScoreThreads / kWave) + w) * 16;
    good[x] = 0;
    if (t < np) {
      const int blk = block_of[min(t + n, np - 1)];
      good[x] = (unsigned)blk < (unsigned)a.NB;
      const size_t unit = (size_t)(good[x] ? blk : 0) * a.H + h;
      const i32x4* m = reinterpret_cast<const i32x4*>(a.means + unit * kHeadDim);
      m0[x] = m[c];
      m1[x] = m[4 + c];
      scale[x] = a.mean_scales[unit];
    }
  }
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const int t = (x * (kScoreThreads / kWave) + w) * 16;
    if (t >= np) continue;
    i32x4 dot = {0, 0, 0, 0};
    dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q0, m0[x], dot, 0, 0, 0);   // rows of the result: query rows, columns: pages
    dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q1, m1[x], dot, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = c * 4 + i;
      if (t + n < np && p0 + t + n < seen[row])
        a.scores[((size_t)(r0 + row) * a.H + h) * a.NP + p0 + t + n] = good[x] ? (float)dot[i] * scale[x] : -INFINITY;
    }
  }
}

// Scores as whole numbers of the same order; -0 does not occur (a product is 0 or at least 2^-126 in magnitude)
__device__ __forceinline__ u32 order_of(float s) {
  const u32 b = as_u32(s);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The k best of a row and head.  Scores are counted in bins of equal width between the least and the largest, which spreads them
// (bins by their bits would not: most scores share a few exponents, and counting them would queue up at a few counters).  The bin
// of the last page that is taken has a few pages then, which are compared with each other; should it have too many (scores that are
// all alike, or have no finite range), their bits are gone through, 11 at a time.  KPT scores of a thread, neighbours.
constexpr int kCandidates = 512;
template <int KPT>
__global__ __launch_bounds__(kSelectThreads) void q8_select_kernel(SelectArgs a) {
  constexpr int NW = kSelectThreads / kWave;
  __shared__ u32 hist[kRadixBins];
  __shared__ int scan[NW + 1];
  __shared__ float least[NW], largest[NW];
  __shared__ u64 cand[kCandidates];
  __shared__ int s_bin, s_below, s_cand;
  const int r = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  int seq;
  const int n = pages_seen(a, r, seq);
  if (n == 0) return;
  const size_t unit = (size_t)r * a.H + h;
  int32_t* out = a.sel + unit * a.k;
  const int want = min(a.k, n);
  for (int i = want + tid; i < a.k; i += kSelectThreads) out[i] = -1;
  if (want == n) {                             // all of them
    for (int i = tid; i < n; i += kSelectThreads) out[i] = i;
    return;
  }
  // (n > k >= sink + recent: the forced pages are different ones)
  const float* s = a.scores + unit * a.NP;
  float v[KPT];
  float lo = INFINITY, hi = -INFINITY;
  auto free_page = [&](int p) { return p < n && p >= a.sink && p < n - a.recent; };
#pragma unroll
  for (int x = 0; x < KPT; ++x) {
    const int p = tid * KPT + x;
    v[x] = p < n ? s[p] : 0.f;
    if (free_page(p) && v[x] > -INFINITY) { lo = fminf(lo, v[x]); hi = fmaxf(hi, v[x]); }
  }
  for (int i = tid; i < kRadixBins; i += kSelectThreads) hist[i] = 0;
  lo = wave_allreduce_min(lo);
  hi = wave_allreduce_max(hi);
  if (tid % kWave == 0) { least[tid / kWave] = lo; largest[tid / kWave] = hi; }
  if (tid == 0) s_cand = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) { lo = fminf(lo, least[i]); hi = fmaxf(hi, largest[i]); }
  const float width = hi - lo;
  const float per = width > 0.f && width < INFINITY ? (kRadixBins - 1) / width : 0.f;
  // (every step of it keeps the order; NaN and what lies outside go to an end)
  auto bin_of = [&](float x) { return (int)fminf(fmaxf((x - lo) * per, 0.f), (float)(kRadixBins - 1)); };
  // the bin, of the counters, that has the need-th item from the top; how many lie above it
  auto find = [&](int need) {
    const int top = kRadixBins - 1 - 2 * tid;  // thread t has bins 2047 - 2 t and the one below
    const int c0 = (int)hist[top], c1 = (int)hist[top - 1];
    int total;
    const int above = block_exclusive_scan<kSelectThreads>(c0 + c1, scan, total);
    if (above < need && need <= above + c0) { s_bin = top; s_below = above; }
    else if (above + c0 < need && need <= above + c0 + c1) { s_bin = top - 1; s_below = above + c0; }
    __syncthreads();
  };
#pragma unroll
  for (int x = 0; x < KPT; ++x)
    if (free_page(tid * KPT + x)) atomicAdd(&hist[bin_of(v[x])], 1u);
  __syncthreads();
  int need = want - min(a.sink, n) - min(a.recent, n);       // of the free pages
  u32 in = 0, in_hi = 0;                       // bit x: page tid * KPT + x is taken
  auto take = [&](int x) { if (x < 32) in |= 1u << x; else in_hi |= 1u << (x - 32); };
  if (need > 0) {
    find(need);
    const int bin = s_bin, count = (int)hist[bin];
    need -= s_below;
    if (count <= kCandidates) {
#pragma unroll
      for (int x = 0; x < KPT; ++x) {
        const int p = tid * KPT + x;
        if (!free_page(p)) continue;
        const int b = bin_of(v[x]);
        if (b > bin) take(x);
        if (b == bin) cand[atomicAdd(&s_cand, 1)] = (u64)order_of(v[x]) << 32 | (u32)~p;   // larger is better
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < KPT; ++x) {
        const int p = tid * KPT + x;
        if (!free_page(p) || bin_of(v[x]) != bin) continue;
        const u64 mine = (u64)order_of(v[x]) << 32 | (u32)~p;
        int better = 0;
        for (int i = 0; i < count; ++i) better += cand[i] > mine;
        if (better < need) take(x);
      }
    } else {
      u32 prefix = 0, mask = 0;
#pragma unroll
      for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const u32 bits = pass == 2 ? 1023u : 2047u;
        __syncthreads();                       // (the counters have been read)
        for (int i = tid; i < kRadixBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < KPT; ++x)
          if (free_page(tid * KPT + x) && bin_of(v[x]) == bin && (order_of(v[x]) & mask) == prefix)
            atomicAdd(&hist[(order_of(v[x]) >> shift) & bits], 1u);
        __syncthreads();
        find(need);
        prefix |= (u32)s_bin << shift;
        mask |= bits << shift;
        need -= s_below;
      }
      // of equal scores the lowest pages
      int same = 0;
#pragma unroll
      for (int x = 0; x < KPT; ++x) same += free_page(tid * KPT + x) && bin_of(v[x]) == bin && order_of(v[x]) == prefix;
      int total;
      int left = need - block_exclusive_scan<kSelectThreads>(same, scan, total);
#pragma unroll
      for (int x = 0; x < KPT; ++x) {
        if (!free_page(tid * KPT + x)) continue;
        const int b = bin_of(v[x]);
        const u32 key = order_of(v[x]);
        if (b > bin || (b == bin && key > prefix)) take(x);
        if (b == bin && key == prefix && left-- > 0) take(x);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < KPT; ++x) {
    const int p = tid * KPT + x;
    if (p < n && !free_page(p)) take(x);
  }
  int total;
  int at = block_exclusive_scan<kSelectThreads>(__popc(in) + __popc(in_hi), scan, total);
#pragma unroll
  for (int x = 0; x < KPT; ++x)
    if ((x < 32 ? in >> x : in_hi >> (x - 32)) & 1) out[at++] = tid * KPT + x;
}

}  // namespace q8
}  // namespace kvd

int64_t kvd_q8_select_bytes(const kvd_q8_cache* c, const kvd_q8_rows* r) {
  return (int64_t)r->n_rows * c->n_kv_heads * r->max_pages * 4;
}

extern "C" int kvd_q8_select(const kvd_q8_cache* c, const kvd_q8_rows* r, const void* q, int64_t q_stride, int32_t* sel_pages,
                             int32_t topk_pages, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace kvd;
  using namespace kvd::q8;
  if (int e = check_cache(c, r)) return e;
  if (topk_pages < 1 || topk_pages > KVD_MAX_TOPK || !stride_ok(q_stride, c->n_q_heads)) return KVD_ERR_SHAPE;
  if ((int64_t)c->sink_pages + c->recent_pages > topk_pages) return KVD_ERR_CAPACITY;
  if (!aligned(c->means, 16) || !aligned(c->mean_scales, 4) || !aligned(q, 16) || !aligned(sel_pages, 4) || !aligned(workspace, 16)) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->row_start, 4) || !aligned(r->row_seq, 4) || !aligned(r->row_pos, 4)) return KVD_ERR_ARG;
  if (workspace_bytes < kvd_q8_select_bytes(c, r)) return KVD_ERR_CAPACITY;
  SelectArgs a;
  a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
  a.table = r->page_table; a.row_start = r->row_start; a.row_seq = r->row_seq; a.row_pos = r->row_pos;
  a.means = c->means; a.mean_scales = c->mean_scales;
  a.scores = static_cast<float*>(workspace); a.sel = sel_pages;
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.H = c->n_kv_heads; a.G = c->n_q_heads / c->n_kv_heads;
  a.P = c->page_size; a.NB = c->n_blocks; a.k = topk_pages; a.sink = c->sink_pages; a.recent = c->recent_pages;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.NP > a.k) {                            // (otherwise no row has more pages than it takes)
    const dim3 grid(a.T, a.H, (a.NP + kScorePages - 1) / kScorePages);
    if (c->kv_dtype == KVD_BF16) hipLaunchKernelGGL(q8_score_kernel<true>, grid, dim3(kScoreThreads), 0, s, a);
    else hipLaunchKernelGGL(q8_score_kernel<false>, grid, dim3(kScoreThreads), 0, s, a);
    if (int e = launched()) return e;
  }
  const dim3 grid(a.T, a.H);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelectThreads), 0, s, a); };
  if (a.NP <= 1024) go(q8_select_kernel<1>);
  else if (a.NP <= 4096) go(q8_select_kernel<4>);
  else if (a.NP <= 8192) go(q8_select_kernel<8>);
  else if (a.NP <= 16384) go(q8_select_kernel<16>);
  else go(q8_select_kernel<64>);
  return launched();
}
