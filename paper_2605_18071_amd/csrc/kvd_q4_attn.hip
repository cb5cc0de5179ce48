// Attention of a step's rows over the pages of the 4-bit cache.
//
// S^T = K Q^T and O^T += V^T P^T on the matrix cores, 128 tokens a wave and step: a result's columns are query rows (a row of the
// step and a head of the group), and the softmaxed S^T of a lane is its operand of the second product, element for element,
// because of the order in which tokens are dealt to the first product's rows.  Codes come from memory in operand order, 16 bytes a lane,
// and become bf16 in registers, which holds every one of them times its scale.  Keys take their scales there.  Values' scales are one
// for 32 elements of a token, which the second product sums over: they go into the weights, so that each group of 32 columns of V has
// weights of its own, p * 2^e.  Where columns would be empty they repeat the rows (REP): each copy weighs the values of a fraction of
// the groups.
//
// (The matrix cores' own products of 4-bit operands with scales take keys and values as they are, but their sums of eight products
// keep 13 bits below the largest: logits of 140 came out 2^-16 off, and small weights beside a large one got lost.)
//
// One pass with a running reference m and sum l of a column: p = 2^(x - m).  m is kHead above the largest logit when it is set, and
// is raised only when a logit passes that by more than kSlack, so that the accumulators are rarely touched; p then stays below
// 2^(kSlack - kHead).  Weights are taken times 2^-kDown, so that those below 2^-4 and values below 2^128 of 2^24 tokens stay finite.
// bf16: they are rounded to bf16, by 2^-8 of themselves at most, like their output.  f16, whose outputs would show it: a
// second product takes what the rounding left (2^-17), and the first one has the queries in two parts of bf16 too.
#include "kvd_q4.h"
#include "kvd_q8_deal.h"

namespace kvd {
namespace q4 {

using q8::deal;
using q8::Unit;
using q8::bf16x8;

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;
constexpr int kAttnGroups = 512;               // workgroups: two for each CU
constexpr int kStep = 8;                       // tiles that a wave takes at a time
constexpr int kLeastTiles = 32;                // tiles of a workgroup at least
constexpr int kColFloats = kHeadDim + 4;       // a column in LDS
// 8-byte words of a partial result: accumulators, then a maximum and a sum a column
__host__ __device__ constexpr size_t part_words(int groups) { return (size_t)groups * (16 * kWave + 16); }
constexpr float kLowest = -3.0e38f, kSlack = 8.f, kHead = 12.f;
constexpr int kDown = 24;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr u32 kNoTile = 0xffffffffu;
using q8::i32x4;

__device__ __forceinline__ i32x4 load_codes(const unsigned char* p) { return __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p)); }
__device__ __forceinline__ i32x4 load_scales(const unsigned char* p) { return *reinterpret_cast<const i32x4*>(p); }

struct AttnArgs {
  const uint16_t* q;
  long long q_stride;
  const int32_t *table, *kv_len, *row_start, *row_from, *prefix_len;
  const float* slopes;
  const unsigned char* pages;
  uint16_t* out;
  float* lse;
  u64* part;
  int32_t* ticket;
  int B, NP, T, H, G, P, NB, R, W, window;
  u32 page_magic;                              // ceil(2^32 / tiles of a page)
  float scale_log2, cap_in, cap_out;           // logits in powers of two: s * scale_log2, or cap_out * tanh(s * cap_in)
};

template <int N, class F>
__device__ __forceinline__ void each_of(F f) {
  if constexpr (N > 0) {
    each_of<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}
__device__ __forceinline__ u64 pack_floats(float a, float b) { return (u64)as_u32(b) << 32 | as_u32(a); }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max_of_column(float x) {      // over the four lanes that have a column
  x = fmaxf(x, __shfl_xor(x, 16, kWave));
  return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Eight codes to an operand, times the scale
__device__ __forceinline__ bf16x8 widen(int codes, float scale) {
  const u32 w = (u32)codes;
  const uint4 x = make_uint4(__builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
  return __builtin_bit_cast(bf16x8, x);
}
// Eight numbers to NP operands: rounded to bf16, and what that left
template <int NP>
__device__ __forceinline__ void parts(const float* x, bf16x8 (&to)[NP]) {
  u32 w[4], rest[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = pack2<true>(x[2 * i], x[2 * i + 1]);
    if (NP > 1) rest[i] = pack2<true>(x[2 * i] - as_f32(w[i] << 16), x[2 * i + 1] - as_f32(w[i] & 0xffff0000u));
  }
  to[0] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
  if constexpr (NP > 1) to[1] = __builtin_bit_cast(bf16x8, make_uint4(rest[0], rest[1], rest[2], rest[3]));
}

template <bool BF16, int NQ, int REP>
struct Wave {
  static constexpr int NP = BF16 ? 1 : 2;      // parts of bf16 that a number of q's type has
  static constexpr int kCols = 16 / REP;       // columns that differ
  static constexpr int kGroups = 4 / REP;      // of V's groups of 32 columns, those that a lane weighs
  static_assert(NQ == 1 || REP == 1, "");
  f32x4 o[NQ][8];
  float m[NQ], l[NQ], slope[NQ];
  bf16x8 q[NQ][4][NP];
  int lo[NQ], hi[NQ], pos[NQ];                 // first and last position that the lane's column sees, its own
  int lo_most, hi_least;                       // what every column sees lies between
  int t_first, t_behind;                       // tiles that any column sees

  const AttnArgs& a;
  const int lane, c, n, tpp;
  Unit u;

  __device__ __forceinline__ Wave(const AttnArgs& a_)
      : a(a_), lane(threadIdx.x % kWave), c((threadIdx.x % kWave) >> 4), n(threadIdx.x & 15), tpp(a_.P / kTile) {}

  // Row of the unit and head of the group of column n + 16 g
  __device__ __forceinline__ void column(int g, int& r, int& head) const {
    const int col = REP > 1 ? n % kCols : n + 16 * g;
    r = col / a.G;
    head = col - r * a.G;
  }
  __device__ __forceinline__ bool real(int r, int head) const { return head < a.G && r < u.rows; }
  // whether this lane's accumulators of 16 columns of V are of the weights that were made for them
  __device__ __forceinline__ bool has(int i) const { return REP == 1 || (i >> 1) % REP == n / kCols; }

  __device__ __forceinline__ void begin(const Unit& unit) {
    u = unit;
    const int len = min(max(a.kv_len[u.seq], 0), a.NP * a.P);
    const int prefix = a.prefix_len ? min(a.prefix_len[u.seq], len) : 0;
    int lo_min = 0x7fffffff, hi_max = -1;
    lo_most = 0;
    hi_least = 0x7fffffff;
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      int r, head;
      column(g, r, head);
      const bool ok = real(r, head);
      const int row = u.row0 + r;
      pos[g] = u.pos0 + r;
      lo[g] = 0x7fffffff;
      hi[g] = -1;
      slope[g] = 0.f;
      uint4 raw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = make_uint4(0, 0, 0, 0);
      if (ok) {
        const uint16_t* src = a.q + (long long)row * a.q_stride + (u.h * a.G + head) * kHeadDim + c * 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const uint4*>(src + i * 8);
        lo[g] = a.window > 0 ? max(pos[g] - a.window + 1, 0) : 0;
        if (a.row_from) lo[g] = max(lo[g], a.row_from[row]);
        hi[g] = min(max(pos[g], prefix - 1), len - 1);
        if (a.slopes) slope[g] = a.slopes[u.h * a.G + head] * kLog2e;
        lo_min = min(lo_min, lo[g]);
        hi_max = max(hi_max, hi[g]);
        lo_most = max(lo_most, lo[g]);
        hi_least = min(hi_least, hi[g]);
      }
      float off = 0.f;                         // a row with an infinity or a NaN gives NaN, and no other row does
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[8];
        cvt8<BF16>(raw[i], f);
#pragma unroll
        for (int y = 0; y < 8; ++y) off += f[y] * 0.f;
        parts<NP>(f, q[g][i]);
      }
      off += __shfl_xor(off, 16, kWave);
      off += __shfl_xor(off, 32, kWave);
      if (off != 0.f)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[g][i][0] = __builtin_bit_cast(bf16x8, make_uint4(~0u, ~0u, ~0u, ~0u));
      m[g] = kLowest;
      l[g] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) {
      lo_min = min(lo_min, __shfl_xor(lo_min, x, kWave));
      lo_most = max(lo_most, __shfl_xor(lo_most, x, kWave));
      hi_max = max(hi_max, __shfl_xor(hi_max, x, kWave));
      hi_least = min(hi_least, __shfl_xor(hi_least, x, kWave));
    }
    t_first = __builtin_amdgcn_readfirstlane(lo_min) / kTile;
    t_behind = (__builtin_amdgcn_readfirstlane(hi_max) + kTile) / kTile;
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);
  }

  // ---- what is on its way

  i32x4 k[8], v[8];
  u32 ks[2];
  i32x4 vs[kGroups][2];
  u32 line, line_next;                         // of the step's tile lane % 8: its place in lines of 128 bytes, or none
  int block_next;                              // of the step after that

  // The block of tile t0 + lane % 8, of those before t1
  __device__ __forceinline__ int block_of(int t0, int t1) const {
    const int t = t0 + (lane & 7);
    int b = -1;
    if (t < t1) {
      const u32 page = tpp == 1 ? t : __umulhi(t, a.page_magic);
      b = a.table[(size_t)u.seq * a.NP + page];
    }
    return b;
  }
  __device__ __forceinline__ u32 line_of(int t0, int b) const {
    const int t = t0 + (lane & 7), sub = tpp == 1 ? 0 : t - (int)__umulhi(t, a.page_magic) * tpp;
    return (unsigned)b < (unsigned)a.NB ? (((u32)b * a.H + u.h) * tpp + sub) * (kTileBytes / 128) : kNoTile;
  }
  // Tile i of the step; the pool's first where there is none (what is read there is hidden)
  __device__ __forceinline__ const unsigned char* tile(u32 lines, int i) const {
    const u32 x = __shfl(lines, i, kWave);
    return a.pages + (size_t)(x == kNoTile ? 0u : x) * 128;
  }
  __device__ __forceinline__ void load_keys(u32 lines) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const unsigned char* at = tile(lines, 2 * (n >> 2) + half) + (n & 3) * 64 + c * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) k[half * 4 + j] = load_codes(at + j * 256);
      ks[half] = *reinterpret_cast<const u32*>(at - (n & 3) * 60 + kKeyScales);
    }
  }
  __device__ __forceinline__ void load_values(u32 lines) {
    const unsigned char *at0 = tile(lines, 2 * c), *at1 = tile(lines, 2 * c + 1);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      v[2 * x] = load_codes(at0 + kValues + n * 16 + x * 256);
      v[2 * x + 1] = load_codes(at1 + kValues + n * 16 + x * 256);
    }
#pragma unroll
    for (int x = 0; x < kGroups; ++x) {
      const int group = x * REP + (REP > 1 ? n / kCols : 0);
      vs[x][0] = load_scales(at0 + kValueScales + group * 16);
      vs[x][1] = load_scales(at1 + kValueScales + group * 16);
    }
  }

  // ---- the step of tiles [t0, t0 + 8)

  // Row r of the products of tile j is token 32 (r / 4) + 4 j + r % 4 of the step, so that lane (c, n) gets tokens 32 c + 0..31 of column n
  __device__ __forceinline__ void scores(f32x4 (&s)[NQ][8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float scale = two_to((int)(ks[j / 4] >> (8 * (j % 4)) & 255) - kBias);
#pragma unroll
      for (int g = 0; g < NQ; ++g) s[g][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 A = widen(k[j][i], scale);
#pragma unroll
        for (int g = 0; g < NQ; ++g)
#pragma unroll
          for (int p = 0; p < NP; ++p) s[g][j] = mfma32(A, q[g][i][p], s[g][j]);
      }
    }
  }
  // Products to logits in powers of two, -infinity where the column does not see the token
  __device__ __forceinline__ void logits(int g, int t0, f32x4 (&s)[8]) {
    const int base = t0 * kTile, at = base + c * 32;
    if (a.cap_in != 0.f) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {          // tanh x = 1 - 2 / (e^2x + 1)
          const float e = __builtin_amdgcn_exp2f(s[j][i] * a.cap_in);
          s[j][i] = a.cap_out - 2.f * a.cap_out * __builtin_amdgcn_rcpf(e + 1.f);
        }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] *= a.scale_log2;
    }
    if (a.slopes) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][i] -= slope[g] * fabsf((float)(pos[g] - (at + j * 4 + i)));
    }
    if (base < lo_most || base + kStep * kTile - 1 > hi_least || __any(line == kNoTile)) {
      const bool none[2] = {__shfl(line, 2 * c, kWave) == kNoTile, __shfl(line, 2 * c + 1, kWave) == kNoTile};
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = at + j * 4 + i;
          if (none[j >> 2] || t < lo[g] || t > hi[g]) s[j][i] = -INFINITY;
        }
    }
  }
  __device__ __forceinline__ void soften(int g, f32x4 (&s)[8], float (&p)[32]) {
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) mx = max3(max3(mx, s[j][0], s[j][1]), s[j][2], s[j][3]);
    if (__any(mx > m[g] - (kHead - kSlack))) {
      mx = max_of_column(mx);
      // (a column that does not need it stays, so that no row's result depends on its neighbours)
      const float to = mx > m[g] - (kHead - kSlack) ? mx + kHead : m[g], down = __builtin_amdgcn_exp2f(m[g] - to);
      m[g] = to;
      l[g] *= down;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[g][i] *= down;
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * j + i] = __builtin_amdgcn_exp2f(s[j][i] - m[g]);
        sum[i] += p[4 * j + i];
      }
    l[g] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // What the tokens add to 32 columns of V (REP > 1: to REP groups of them, of which one has this lane's weights)
  template <int X>
  __device__ __forceinline__ void weigh(const float (&p)[NQ][32]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {              // eight of the lane's tokens
      bf16x8 B[NQ][NP];
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        float w[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const u32 word = vs[X][i >> 1][(i & 1) * 2 + (y >> 2)];
          w[y] = __builtin_amdgcn_ldexpf(p[g][8 * i + y], (int)(word >> (8 * (y & 3)) & 255) - (kBias + kDown));
        }
        parts<NP>(w, B[g]);
      }
#pragma unroll
      for (int z = 0; z < 2 * REP; ++z) {
        const int d = X * 2 * REP + z;         // 16 columns
        const bf16x8 A = widen(v[d / 2 * 2 + (i >> 1)][d % 2 * 2 + (i & 1)], 1.f);
#pragma unroll
        for (int g = 0; g < NQ; ++g)
#pragma unroll
          for (int y = 0; y < NP; ++y) o[g][d] = mfma32(A, B[g][y], o[g][d]);
      }
    }
  }

  // Tiles [from, to) of the unit.  Keys of the next step are asked for when those of this one have been taken, values likewise;
  // the blocks of the tiles two steps ahead.
  __device__ __forceinline__ void sweep(int from, int to) {
    if (from < to) {
      line = line_of(from, block_of(from, to));
      block_next = block_of(from + kStep, to);
      load_keys(line);
      load_values(line);
      for (int t = from; t < to; t += kStep) {
        const bool more = t + kStep < to;
        f32x4 s[NQ][8];
        scores(s);
        if (more) {
          __builtin_amdgcn_sched_barrier(0);
          line_next = line_of(t + kStep, block_next);
          block_next = block_of(t + 2 * kStep, to);
          load_keys(line_next);
          __builtin_amdgcn_sched_barrier(0);
        }
        float p[NQ][32];
#pragma unroll
        for (int g = 0; g < NQ; ++g) {
          logits(g, t, s[g]);
          soften(g, s[g], p[g]);
        }
        each_of<kGroups>([&](auto x) { weigh<decltype(x)::value>(p); });
        if (more) {
          __builtin_amdgcn_sched_barrier(0);
          line = line_next;
          load_values(line);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    // a column's four lanes have a quarter of its sum each
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      l[g] += __shfl_xor(l[g], 16, kWave);
      l[g] += __shfl_xor(l[g], 32, kWave);
    }
  }

  // Partial results of other workgroups, as this launch's lanes have them: accumulators [g][i][half][lane] in pairs, then
  // (maximum, sum) [g][n]
  __device__ __forceinline__ u64* part_of(int slot) const { return a.part + (size_t)slot * part_words(NQ); }
  // Lane that has column n's accumulators of 16 columns of V
  __device__ __forceinline__ int lane_of(int i, int col, int quarter) const { return quarter * 16 + (REP == 1 ? col : col % kCols + (i >> 1) % REP * kCols); }

  // The joined results slot(from), slot(from + step), ... of `count`
  template <class Slot>
  __device__ __forceinline__ void gather(int from, int step, int count, Slot slot) {
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      m[g] = kLowest;
      l[g] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int x = from; x < count; x += step) {
      const u64* part = part_of(slot(x));
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        const u64 ml = load_agent(part + NQ * 16 * kWave + g * 16 + n % kCols);
        u64 y[8][2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i][0] = load_agent(part + (g * 8 + i) * 2 * kWave + lane_of(i, n, c));
          y[i][1] = load_agent(part + ((g * 8 + i) * 2 + 1) * kWave + lane_of(i, n, c));
        }
        const float l2 = as_f32((u32)(ml >> 32)), m2 = l2 == 0.f ? kLowest : as_f32((u32)ml);
        const float to = fmaxf(m[g], m2), f1 = __builtin_amdgcn_exp2f(m[g] - to), f2 = l2 == 0.f ? 0.f : __builtin_amdgcn_exp2f(m2 - to);
        m[g] = to;
        l[g] = l[g] * f1 + l2 * f2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const f32x4 z = {as_f32((u32)y[i][0]), as_f32((u32)(y[i][0] >> 32)), as_f32((u32)y[i][1]), as_f32((u32)(y[i][1] >> 32))};
          o[g][i] = o[g][i] * f1 + z * f2;
        }
      }
    }
  }
};

// A column's result over all tokens
template <bool BF16, int N>
__device__ __forceinline__ void emit(const AttnArgs& a, const Unit& u, int r, int head, int d, const float (&v)[N], float m, float l) {
  const size_t at = (size_t)(u.row0 + r) * a.H * a.G + u.h * a.G + head;
  const float inv = l == 0.f ? 0.f : two_to(kDown) / l;
  u32 w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = pack2<BF16>(l == 0.f ? 0.f : v[2 * i] * inv, l == 0.f ? 0.f : v[2 * i + 1] * inv);
  if constexpr (N == 8) *reinterpret_cast<uint4*>(a.out + at * kHeadDim + d) = make_uint4(w[0], w[1], w[2], w[3]);
  else *reinterpret_cast<uint2*>(a.out + at * kHeadDim + d) = make_uint2(w[0], w[1]);
  if (a.lse != nullptr && d == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int NQ>
struct AttnLds {
  float ml[kAttnWaves][16 * NQ][2];
  __align__(16) float o[kAttnWaves][16][kColFloats];
  int last;
};

// The waves' results of one unit as one: with to_slot < 0 to the output, else there
template <bool BF16, int NQ, int REP>
__device__ __forceinline__ void merge_waves(const AttnArgs& a, const Wave<BF16, NQ, REP>& w, AttnLds<NQ>& lds, int to_slot) {
  typedef Wave<BF16, NQ, REP> W;
  const int tid = threadIdx.x, wave = tid / kWave;
  __syncthreads();                             // (what was there has been read)
#pragma unroll
  for (int g = 0; g < NQ; ++g)
    if (w.c == 0) {
      lds.ml[wave][g * 16 + w.n][0] = w.l[g] == 0.f ? kLowest : w.m[g];
      lds.ml[wave][g * 16 + w.n][1] = w.l[g];
    }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < NQ; ++g) {
    float M = kLowest;
#pragma unroll
    for (int i = 0; i < kAttnWaves; ++i) M = fmaxf(M, lds.ml[i][g * 16 + w.n][0]);
    const float f = w.l[g] == 0.f ? 0.f : __builtin_amdgcn_exp2f(w.m[g] - M);
    if (g > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (w.has(i)) *reinterpret_cast<f32x4*>(&lds.o[wave][w.n % W::kCols][i * 16 + w.c * 4]) = w.o[g][i] * f;
    __syncthreads();
    const int n = tid >> 4, d = (tid & 15) * 8;   // a column and eight of its elements
    const int col = g * 16 + n, r = col / a.G, head = col - r * a.G;
    if (n < W::kCols && w.real(r, head)) {
      float top = kLowest, L = 0.f, v[8];
#pragma unroll
      for (int i = 0; i < kAttnWaves; ++i) top = fmaxf(top, lds.ml[i][col][0]);
#pragma unroll
      for (int i = 0; i < kAttnWaves; ++i) {
        const float l = lds.ml[i][col][1];
        if (l != 0.f) L += l * __builtin_amdgcn_exp2f(lds.ml[i][col][0] - top);
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        v[y] = 0.f;
#pragma unroll
        for (int i = 0; i < kAttnWaves; ++i) v[y] += lds.o[i][n][d + y];
      }
      if (to_slot < 0) emit<BF16>(a, w.u, r, head, d, v, top, L);
      else {
        u64* part = w.part_of(to_slot);
        const int i = d / 16, at = (g * 8 + i) * 2 * kWave;
#pragma unroll
        for (int y = 0; y < 4; ++y)
          store_agent(part + at + (y & 1) * kWave + w.lane_of(i, n, d % 16 / 4 + (y >> 1)), pack_floats(v[2 * y], v[2 * y + 1]));
        if (d == 0) store_agent(part + NQ * 16 * kWave + col, pack_floats(top, L));
      }
    }
  }
}

// Tiles [t0, t1) of a unit: by all waves, or, if they are one step, by wave `solo` alone.  Its result goes to the output if it is all of the
// unit (count == 1), else to slot `mine` of the partial results, which the last of the `count` pieces to arrive joins, in
// their order; slot(i) is the i-th one's number.
template <bool BF16, int NQ, int REP, class Slot>
__device__ __forceinline__ void piece(const AttnArgs& a, Wave<BF16, NQ, REP>& w, AttnLds<NQ>& lds, const Unit& u, int t0, int t1,
                                      int solo, int count, int mine, int ticket, Slot slot) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const bool alone = count == 1 && t1 - t0 <= kStep;   // (pieces of one unit are joined in one way, whichever comes last: the sums' order is fixed)
  if (alone && wave != solo) return;
  w.begin(u);
  t0 = max(t0, w.t_first);
  t1 = max(min(t1, w.t_behind), t0);
  if (!alone) {
    const int per = ((t1 - t0 + kStep - 1) / kStep + kAttnWaves - 1) / kAttnWaves * kStep;
    t0 = min(t0 + wave * per, t1);
    t1 = min(t0 + per, t1);
  }
  w.sweep(t0, t1);
  if (alone) {
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      int r, head;
      w.column(g, r, head);
      if (!w.real(r, head)) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (!w.has(i)) continue;
        const float v[4] = {w.o[g][i][0], w.o[g][i][1], w.o[g][i][2], w.o[g][i][3]};
        emit<BF16>(a, u, r, head, i * 16 + w.c * 4, v, w.m[g], w.l[g]);
      }
    }
    return;
  }
  merge_waves(a, w, lds, count == 1 ? -1 : mine);
  if (count == 1) return;
  wave_drain_memory();                         // (written through and drained before the ticket, and read past the caches)
  __syncthreads();
  if (threadIdx.x == 0) {
    lds.last = __hip_atomic_fetch_add(a.ticket + ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1;
    if (lds.last) store_agent(a.ticket + ticket, 0);
  }
  __syncthreads();
  if (!lds.last) return;
  w.gather(wave, kAttnWaves, count, slot);
  merge_waves(a, w, lds, -1);
}

template <bool BF16, int NQ, int REP>
__global__ __launch_bounds__(kAttnThreads, NQ == 2 ? 1 : 2) void q4_attn_kernel(AttnArgs a) {
  __shared__ AttnLds<NQ> lds;
  Wave<BF16, NQ, REP> w(a);
  int solo = 0;
  // what a window leaves of a unit begins at the tile of the first position that its first row sees
  const bool windowed = a.window > 0 && a.prefix_len == nullptr;
  const int most = windowed ? (int)min(((long long)a.window + a.R + 2 * kTile - 3) / kTile, (long long)q8::kAllTiles) : q8::kAllTiles;
  deal<kAttnThreads, kLeastTiles>(a, false, most, [&](const Unit& u, int t0, int t1, int f, int count, int mine, auto slot) {
    const int first = windowed ? max(u.pos0 - a.window + 1, 0) / kTile : 0;
    piece(a, w, lds, u, first + t0, first + t1, solo, count, mine, f, slot);
    solo = (solo + 1) % kAttnWaves;
  });
}

// Columns of 16 that the rows of a unit take, and how often they are repeated
struct Shape { int groups, copies; };
static Shape shape_of(int T, int B, int G) {
  const int64_t want = (int64_t)((T + B - 1) / B) * G;
  return {want > 16 ? 2 : 1, want <= 4 ? 4 : want <= 8 ? 2 : 1};
}

}  // namespace q4
}  // namespace kvd

extern "C" int64_t kvd_q4_workspace_bytes(const kvd_q4_cache* c, const kvd_q8_rows* r) {
  using namespace kvd::q4;
  if (int e = check_cache(c, r)) return e;
  static_assert(kAttnGroups * 4 <= kvd::q8::kTicketBytes, "a ticket for each workgroup");
  return kvd::q8::kTicketBytes + (int64_t)kAttnGroups * 2 * 8 * part_words(shape_of(r->n_rows, r->n_seqs, c->n_q_heads / c->n_kv_heads).groups);
}

extern "C" int kvd_q4_attn(const kvd_q4_cache* c, const kvd_q8_rows* r, const void* q, int64_t q_stride, const kvd_q4_scores* f,
                           void* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace kvd::q4;
  using kvd::kHeadDim;
  if (int e = check_cache(c, r)) return e;
  if (!stride_ok(q_stride, c->n_q_heads)) return KVD_ERR_SHAPE;
  if (!aligned(c->pages, 128) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16)) return KVD_ERR_ARG;
  if (out == q) return KVD_ERR_ARG;            // (a row's pieces read q while the first unit that is done writes)
  if (reinterpret_cast<uintptr_t>(lse) & 3) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->kv_len, 4) || !aligned(r->row_start, 4)) return KVD_ERR_ARG;
  AttnArgs a = {};
  a.scale_log2 = (c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e;
  if (f) {
    if (!(f->softcap >= 0.f) || isinf(f->softcap)) return KVD_ERR_ARG;
    if (f->window < 0) return KVD_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(f->slopes) | reinterpret_cast<uintptr_t>(f->row_from) | reinterpret_cast<uintptr_t>(f->prefix_len)) & 3)
      return KVD_ERR_ARG;
    if (f->softcap > 0.f) {
      a.cap_in = 2.f * a.scale_log2 / f->softcap;
      a.cap_out = f->softcap * kLog2e;
      if (!(a.cap_in > 0.f) || isinf(a.cap_in) || isinf(a.cap_out)) return KVD_ERR_ARG;
    }
    a.window = f->window; a.slopes = f->slopes; a.row_from = f->row_from; a.prefix_len = f->prefix_len;
  }
  if (workspace_bytes < kvd_q4_workspace_bytes(c, r)) return KVD_ERR_CAPACITY;
  a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
  a.table = r->page_table; a.kv_len = r->kv_len; a.row_start = r->row_start;
  a.pages = static_cast<const unsigned char*>(c->pages);
  a.out = static_cast<uint16_t*>(out); a.lse = lse;
  a.ticket = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<kvd::u64*>(static_cast<char*>(workspace) + kvd::q8::kTicketBytes);
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.H = c->n_kv_heads; a.G = c->n_q_heads / c->n_kv_heads;
  a.P = c->page_size; a.NB = c->n_blocks;
  a.W = kAttnGroups;
  const int tpp = a.P / kTile;
  a.page_magic = (kvd::u32)(((1ull << 32) + tpp - 1) / tpp);
  const Shape shape = shape_of(a.T, a.B, a.G);
  a.R = 16 * shape.groups / shape.copies / a.G;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.W), dim3(kAttnThreads), 0, s, a); };
  if (c->kv_dtype == KVD_BF16) {
    if (shape.groups == 2) go(q4_attn_kernel<true, 2, 1>);
    else if (shape.copies == 4) go(q4_attn_kernel<true, 1, 4>);
    else if (shape.copies == 2) go(q4_attn_kernel<true, 1, 2>);
    else go(q4_attn_kernel<true, 1, 1>);
  } else {
    if (shape.groups == 2) go(q4_attn_kernel<false, 2, 1>);
    else if (shape.copies == 4) go(q4_attn_kernel<false, 1, 4>);
    else if (shape.copies == 2) go(q4_attn_kernel<false, 1, 2>);
    else go(q4_attn_kernel<false, 1, 1>);
  }
  return launched();
}
