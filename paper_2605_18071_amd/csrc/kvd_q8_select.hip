// Selection of pages by a score in 8 bits.  Two launches: the scores of all visible pages of every row and head, as
// products of whole numbers (int8, exact, so that the result does not depend on the order), and the k best
// of a row and head by one workgroup, which holds the scores in registers (a table of more than 16384 pages has 64 a
// thread, of which the compiler spills about half).  Scoring is bound by the memory (132 bytes a page and
// head), selecting by its trips to LDS.
#include <type_traits>

#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kScoreThreads = 256;
constexpr int kFewGroups = 512;                // workgroups below which a wave takes fewer pages: two for each CU
constexpr int kScoreGroups = 768;              // workgroups from which on one takes several times that: three for each CU
constexpr int kScoreRows = 16;                 // rows of one sequence that share its reading of the index
constexpr int kSelectThreads = 1024;

struct SelectArgs {
  const uint16_t* q;
  long long q_stride;
  const int32_t *table, *row_seq, *row_pos;
  const int8_t* means;
  const float* mean_scales;
  float* scores;                               // [T][H][NP]
  int32_t* sel;
  int B, NP, T, H, G, P, NB, k, sink, recent, span;
};

// Pages that row r sees, 0 where it has no sequence or a position outside its table
__device__ __forceinline__ int pages_seen(const SelectArgs& a, int r, int& seq) {
  seq = a.row_seq[r];
  const int pos = a.row_pos[r];
  if ((unsigned)seq >= (unsigned)a.B || pos < 0 || pos >= a.NP * a.P) return 0;
  return pos / a.P + 1;
}

// One workgroup: up to 16 rows of a sequence and HG heads, PW pages a wave and step (64, and less where that would leave CUs without
// work: 12 x 4 rows of 938 pages take 15 us with 64).  A load takes the entries of all these heads from one
// page (8 lanes of 16 bytes a head): they are neighbours in memory, and a load whose lanes went to 16 pages, as operands of the
// matrix cores would have it, went at 3.1 TB/s instead of 4.5 (31 us for 16 x 8192 pages of 8 heads).
// The products are few enough for the vector unit: four elements an instruction.
template <bool BF16, int HG, int PW>
__global__ __launch_bounds__(kScoreThreads, 4) void q8_score_kernel(SelectArgs a) {
  constexpr int kPages = 8 / HG;               // of a load
  constexpr int kScorePages = kScoreThreads / kWave * PW;
  __shared__ __align__(16) int8_t qi[HG][kScoreRows][kHeadDim];
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const int sub = lane / (8 * HG), x = lane / 8 % HG, k = lane % 8;          // page of the load, head, 16 elements
  const int span = a.span * kScorePages;       // pages of this workgroup
  const int r0 = blockIdx.x, h0 = blockIdx.y * HG, p0 = blockIdx.z * span;
  const bool head = h0 + x < a.H;
  // rows r0 .. up to the next multiple of 16, as far as they are of one sequence; lanes 16 apart have the same
  const int n = lane & 15, r = min(r0 + n, a.T - 1), row_seq = a.row_seq[r], row_pos = a.row_pos[r];
  const int before = r0 % kScoreRows ? a.row_seq[r0 - 1] : -1;
  const int seq = __builtin_amdgcn_readfirstlane(row_seq);
  if ((unsigned)seq >= (unsigned)a.B) return;
  const bool mine = row_seq == seq && r0 % kScoreRows + n < kScoreRows && r0 + n < a.T && row_pos >= 0 && row_pos < a.NP * a.P;
  const int seen = mine ? row_pos / a.P + 1 : 0;
  int most = seen;
#pragma unroll
  for (int y = 8; y >= 1; y >>= 1) most = max(most, __shfl_xor(most, y, kWave));
  most = __builtin_amdgcn_readfirstlane(most);
  if (p0 >= most) return;
  const int np = min(most - p0, span);
  const int32_t* table = a.table + (size_t)seq * a.NP + p0;
  auto blocks_of = [&](int at) { return lane < PW && at + lane < np ? table[at + lane] : -1; };   // of the wave's pages from `at` on
  int at = w * PW;
  int blk = blocks_of(at);
  if (before == seq) return;                   // (an earlier row's workgroup has this one, too)
  // the queries in 8 bits: a wave a row and head, two elements a lane
  for (int i = w; i < kScoreRows * HG; i += kScoreThreads / kWave) {
    const int row = i / HG, y = i % HG;
    if (h0 + y >= a.H || __builtin_amdgcn_readlane(seen, row) == 0) continue;
    const uint16_t* q = a.q + (long long)(r0 + row) * a.q_stride + (h0 + y) * a.G * kHeadDim + lane * 2;
    u32 raw[KVD_MAX_GROUP];
#pragma unroll
    for (int g = 0; g < KVD_MAX_GROUP; ++g) raw[g] = g < a.G ? *reinterpret_cast<const u32*>(q + g * kHeadDim) : 0;
    double s0 = 0.0, s1 = 0.0;
#pragma unroll
    for (int g = 0; g < KVD_MAX_GROUP; ++g) {
      if (BF16) { s0 += (double)as_f32(raw[g] << 16); s1 += (double)as_f32(raw[g] & 0xffff0000u); }
      else { const f16x2 v = __builtin_bit_cast(f16x2, raw[g]); s0 += (double)(float)v.x; s1 += (double)(float)v.y; }
    }
    double m = fmax(fabs(s0), fabs(s1));
#pragma unroll
    for (int z = 32; z >= 1; z >>= 1) m = fmax(m, __shfl_xor(m, z, kWave));
    const double inv = 127.0 / m;
    const double a0 = s0 * inv, a1 = s1 * inv;
    const int i0 = fabs(a0) < 128.0 ? (int)rint(a0) : 0, i1 = fabs(a1) < 128.0 ? (int)rint(a1) : 0;     // (not for NaN)
    *reinterpret_cast<uint16_t*>(&qi[y][row][lane * 2]) = (uint16_t)((i0 & 0xff) | (i1 & 0xff) << 8);
  }
  __syncthreads();
  // eight loads at a time
  i32x4 m[2][8];
  float scale[2][8];
  auto ask = [&](int blocks, int first, i32x4 (&v)[8], float (&f)[8]) {        // pages first .. of those whose blocks these are
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int b = __shfl(blocks, first + i * kPages + sub, kWave);
      v[i] = i32x4{0, 0, 0, 0};
      f[i] = -1.f;                             // a bad block
      if (head && (unsigned)b < (unsigned)a.NB) {
        const size_t unit = (size_t)b * a.H + h0 + x;
        v[i] = *reinterpret_cast<const i32x4*>(a.means + unit * kHeadDim + k * 16);
        f[i] = a.mean_scales[unit];
      }
    }
  };
  auto take = [&](int first, const i32x4 (&v)[8], const float (&f)[8]) {
    for (int row = 0; row < kScoreRows; ++row) {
      const int sees = __builtin_amdgcn_readlane(seen, row);
      if (sees == 0) continue;
      const i32x4 q = *reinterpret_cast<const i32x4*>(&qi[x][row][k * 16]);
      float score = 0.f;                       // of load k's page: every one of the eight lanes keeps one
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int dot = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) dot = __builtin_amdgcn_sdot4(v[i][y], q[y], dot, false);
        dot += __builtin_amdgcn_update_dpp(0, dot, 0xb1, 0xf, 0xf, true);    // quad_perm 1 0 3 2
        dot += __builtin_amdgcn_update_dpp(0, dot, 0x4e, 0xf, 0xf, true);    // quad_perm 2 3 0 1
        dot += __builtin_amdgcn_update_dpp(0, dot, 0x141, 0xf, 0xf, true);   // row_half_mirror: the other four of eight lanes
        const float y = f[i] >= 0.f ? (float)dot * f[i] : -INFINITY;
        if (k == i) score = y;
      }
      const int p = first + k * kPages + sub;
      if (head && p < np && p0 + p < sees) a.scores[((size_t)(r0 + row) * a.H + h0 + x) * a.NP + p0 + p] = score;
    }
  };
  constexpr int kStep = 8 * kPages;            // pages of eight loads: 8 to 64
  if (at < np) ask(blk, 0, m[0], scale[0]);
  for (; at < np; at += kScorePages) {
    const int next = blocks_of(at + kScorePages);
#pragma unroll
    for (int i = 0; i < PW; i += 2 * kStep) {  // (a step of all of them: what would be its second half is the next round's first)
      if constexpr (kStep < PW) {
        ask(blk, i + kStep, m[1], scale[1]);
        take(at + i, m[0], scale[0]);
        if (i + 2 * kStep < PW) ask(blk, i + 2 * kStep, m[0], scale[0]);
        else ask(next, 0, m[0], scale[0]);
        take(at + i + kStep, m[1], scale[1]);
      } else {
        take(at, m[0], scale[0]);
        ask(next, 0, m[0], scale[0]);
      }
    }
    blk = next;
  }
}

// Scores as whole numbers of the same order; -0, which a scale of 0 makes of a negative product, is 0
__device__ __forceinline__ u32 order_of(float s) {
  const u32 b = as_u32(s + 0.f);
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
  return kvd::q8::kTicketBytes + (int64_t)r->n_rows * c->n_kv_heads * r->max_pages * 4;
}

extern "C" int kvd_q8_select(const kvd_q8_cache* c, const kvd_q8_rows* r, const void* q, int64_t q_stride, int32_t* sel_pages,
                             int32_t topk_pages, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace kvd;
  using namespace kvd::q8;
  if (int e = check_cache(c, r)) return e;
  if (topk_pages < 1 || topk_pages > KVD_MAX_TOPK || !stride_ok(q_stride, c->n_q_heads)) return KVD_ERR_SHAPE;
  if ((int64_t)c->sink_pages + c->recent_pages > topk_pages) return KVD_ERR_CAPACITY;
  if (!aligned(c->means, 16) || !aligned(c->mean_scales, 4) || !aligned(q, 16) || !aligned(sel_pages, 4) || !aligned(workspace, 16)) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->row_seq, 4) || !aligned(r->row_pos, 4)) return KVD_ERR_ARG;
  if (workspace_bytes < kvd_q8_select_bytes(c, r)) return KVD_ERR_CAPACITY;
  SelectArgs a;
  a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
  a.table = r->page_table; a.row_seq = r->row_seq; a.row_pos = r->row_pos;
  a.means = c->means; a.mean_scales = c->mean_scales;
  a.scores = reinterpret_cast<float*>(static_cast<char*>(workspace) + kTicketBytes); a.sel = sel_pages;
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.H = c->n_kv_heads; a.G = c->n_q_heads / c->n_kv_heads;
  a.P = c->page_size; a.NB = c->n_blocks; a.k = topk_pages; a.sink = c->sink_pages; a.recent = c->recent_pages;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.NP > a.k) {                            // (otherwise no row has more pages than it takes)
    // (a grid's first dimension holds the rows, its third at most 1024 workgroups)
    const int heads = a.H >= 5 ? 8 : a.H >= 3 ? 4 : a.H;
    const int head_groups = (a.H + heads - 1) / heads;
    auto steps = [&](int pages) { return (a.NP + pages - 1) / pages; };       // of a workgroup
    const bool few = (int64_t)a.T * head_groups * steps(kScoreThreads) < kFewGroups;
    const int pages = kScoreThreads / kWave * (few ? heads == 1 ? 64 : heads == 2 ? 32 : 16 : 64);
    const int64_t most = (int64_t)a.T * head_groups * steps(pages);
    const int64_t span = most / kScoreGroups;
    a.span = few || span < 1 ? 1 : span > 16 ? 16 : (int)span;
    const dim3 grid(a.T, head_groups, (steps(pages) + a.span - 1) / a.span);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kScoreThreads), 0, s, a); };
    auto go_type = [&](auto type) {
      constexpr bool BF16 = decltype(type)::value;
      if (heads == 8) { if (few) go(q8_score_kernel<BF16, 8, 16>); else go(q8_score_kernel<BF16, 8, 64>); }
      else if (heads == 4) { if (few) go(q8_score_kernel<BF16, 4, 16>); else go(q8_score_kernel<BF16, 4, 64>); }
      else if (heads == 2) { if (few) go(q8_score_kernel<BF16, 2, 32>); else go(q8_score_kernel<BF16, 2, 64>); }
      else go(q8_score_kernel<BF16, 1, 64>);
    };
    if (c->kv_dtype == KVD_BF16) go_type(std::true_type{});
    else go_type(std::false_type{});
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
