// Attention of a step's rows over the pages of the 4-bit cache.
//
// S^T = K Q^T and O^T += V^T P^T on the matrix cores: a result's columns are query rows (a row of the step and a head of the group),
// and the softmaxed S^T of a lane is its operand of the second product, element for element, because of the order in which
// tokens are dealt to the first product's rows.  Codes come from memory in operand order, 16 bytes a lane, and become bf16 in
// registers, which holds every one of them times its scale.
//
// (The matrix cores' own products of 4-bit operands with scales take keys and values as they are, but their sums of eight products
// keep 13 bits below the largest: logits of 140 came out 2^-16 off, and small weights beside a large one got lost.)
//
// One pass with a running reference m and sum l of a column: p = 2^(x - m).  m is HEAD above the largest logit when it is set, and
// is raised only when a logit passes that by more than kSlack, so that the accumulators are rarely touched.  What multiplies values
// of up to 2^128 stays below 2^-28, so that 2^24 of them have finite sums.
// Weights have 16 bits: a second product takes what rounding them to bf16 left, which is off by 2^-16 of a weight at most.  (Without it
// outputs in bf16 are off by 2.1e-3 to 2.3e-3 of their norm instead of the 1.6e-3 of their own rounding, and it is 100 us for 104 at 16 x
// 32768 tokens, 11.3 for 12.2 where contexts are short, 513 for 665 where rows are many.)  f16 has the queries in two parts of bf16 too.
#include "kvd_q4.h"
#include "kvd_q8_deal.h"

namespace kvd {
namespace q4 {

using q8::bf16x8;
using q8::deal;
using q8::i32x4;
using q8::Unit;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;
constexpr int kAttnGroups = 512;               // workgroups: two for each CU
constexpr int kStep = 8;                       // tiles that a wave takes at a time
constexpr int kLeastTiles = 32;                // tiles of a workgroup at least
// What a unit costs whatever its length, in tiles: without it the workgroups that have many short units come last (2 x 4096 rows from
// the start 510 us for 440, 24 drafts of ragged contexts 118 for 116)
constexpr int kFewPad = 16, kRowsPad = 24;
// Tiles of a workgroup where there are few, so that most units need no joining: 30 contexts of up to 3000 tokens of 8 heads 22 us; with 32
// 28, with 128 27.  4 x 2500: 14.9, 14.0, 18.2
constexpr int kPieceTiles = 64;
// What becomes of logits, in kernels of their own (a branch for large caps in the ones without: f16 drafts 136 us for 123)
constexpr int kPlain = 0, kShaped = 1, kShapedFar = 2;         // nothing; a cap, slopes; a cap above kNearCap, slopes
constexpr float kNearCap = 64;                 // up to here a cap's logits are off by 2^-20 of the cap, beyond it by 2^-20 of themselves
constexpr int kColFloats = kHeadDim + 4;       // a column in LDS
constexpr int kPartWords = 16 * kWave + 16;    // 8-byte words of 16 columns' partial result: accumulators, then a maximum and a sum a column
constexpr int kWeightParts = 2;                // operands of bf16 that a weight has: rounded, or cut, and what that left
constexpr float kLowest = -3.0e38f, kSlack = 8.f;
constexpr int kFewHead = -90, kRowsHead = 36, kFewDown = 126;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr u32 kNoTile = 0xffffffffu;

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
  u32 page_magic;                              // ceil(2^32 / tiles of a page), for pages of several
  float scale_log2, cap_in, cap_out;           // logits in powers of two: s * scale_log2, or cap_out * tanh(s * cap_in * ln 2 / 2); 0: no cap
};

template <int N, class F>
__device__ __forceinline__ void each_of(F f) {
  if constexpr (N > 0) {
    each_of<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}
template <bool ONCE>                           // whether no other wave of the workgroup reads them
__device__ __forceinline__ i32x4 load_codes(const unsigned char* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p));
  else return *reinterpret_cast<const i32x4*>(p);
}
__device__ __forceinline__ i32x4 load_scales(const unsigned char* p) { return *reinterpret_cast<const i32x4*>(p); }
__device__ __forceinline__ u64 pack_floats(float a, float b) { return (u64)as_u32(b) << 32 | as_u32(a); }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max_of_column(float x) {      // over the four lanes that have a column
  x = fmaxf(x, __shfl_xor(x, 16, kWave));
  return fmaxf(x, __shfl_xor(x, 32, kWave));
}
__device__ __forceinline__ float sum_of_column(float x) {
  x += __shfl_xor(x, 16, kWave);
  return x + __shfl_xor(x, 32, kWave);
}
__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ u32 byte_of(u32 w, int i) { return w >> (8 * i) & 255; }

// tanh(x ln 2 / 2) / 2, off by 2^-21 of itself, where a cap is so large that 2^-24 of it would show.  Near 0 by its continued fraction
// y / (1 + y^2 / (3 + y^2 / (5 + y^2 / (7 + y^2 / 9)))), off by y^10 / 9823275 of itself: below 2^-27 where it is taken
__device__ __forceinline__ float half_tanh(float x) {
  const float y = x * (kLn2 / 2), z = y * y;
  const float near = y * 0.5f * (945.f + z * (105.f + z)) * __builtin_amdgcn_rcpf(945.f + z * (420.f + z * 15.f));
  return fabsf(y) < 0.75f ? near : 0.5f + __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(x));
}
// Eight codes to an operand, times the scale
__device__ __forceinline__ bf16x8 widen(int codes, float scale) {
  const u32 w = (u32)codes;
  const uint4 x = make_uint4(__builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                             __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
  return __builtin_bit_cast(bf16x8, x);
}
// The two codes of byte BYTE, times a scale each
template <int BYTE>
__device__ __forceinline__ u32 pair(u32 codes, float first, float second) {
  const u32 lo = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, first, BYTE));
  const u32 hi = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, second, BYTE));
  return (lo & 0xffffu) | (hi & 0xffff0000u);
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

// a * b + c of two 16-bit whole numbers each (which the compiler would take apart where b is a power of two)
__device__ __forceinline__ u16x2 mad_pair(u32 a, u32 b, u32 c) {
  u32 x;
  asm("v_pk_mad_u16 %0, %1, %2, %3" : "=v"(x) : "v"(a), "s"(b), "v"(c));
  return __builtin_bit_cast(u16x2, x);
}
// Eight weights, none of them negative, to operands whose parts are not negative either: cut to bf16, and what that left, rounded: off by
// 2^-16 of themselves at most
__device__ __forceinline__ void weights(const float* p, u16x2 (&to)[kWeightParts][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = p[2 * i], b = p[2 * i + 1];
    to[0][i] = __builtin_bit_cast(u16x2, __builtin_amdgcn_perm(as_u32(b), as_u32(a), 0x07060302));
    to[1][i] = __builtin_bit_cast(u16x2, pack2<true>(a - as_f32(as_u32(a) & 0xffff0000u), b - as_f32(as_u32(b) & 0xffff0000u)));
  }
}

// What any and what every column of a wave sees
struct Seen {
  int first, behind;                           // tiles that any column sees
  int lo, hi;                                  // positions that every column sees
};

// Sixteen columns: lane (c, n) = (lane / 16, lane % 16) has elements 16 i + 4 c + 0..3 of column n in o[i]
template <bool BF16, int SHAPE, int HEAD>
struct Columns {
  static constexpr float kHead = HEAD;
  static constexpr int NP = BF16 ? 1 : 2;      // parts of bf16 that a number of q's type has
  f32x4 o[8];
  float m, l, slope;
  int lo, hi, pos;                             // first and last position that the lane's column sees, its own
  bf16x8 q[4][NP];                             // elements 32 c + 8 i + 0..7

  __device__ __forceinline__ void clear() {
    m = kLowest;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // Row r of the unit and head of its group, or (!ok) a column that is none
  __device__ __forceinline__ void begin(const AttnArgs& a, const Unit& u, bool ok, int r, int head, int len, int prefix, int (&see)[4]) {
    const int row = u.row0 + r;
    pos = u.pos0 + r;
    lo = 0x7fffffff;
    hi = -1;
    slope = 0.f;
    uint4 raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = make_uint4(0, 0, 0, 0);
    if (ok) {
      const uint16_t* src = a.q + (long long)row * a.q_stride + (u.h * a.G + head) * kHeadDim + (threadIdx.x % kWave >> 4) * 32;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const uint4*>(src + i * 8);
      lo = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
      if (a.row_from) lo = max(lo, a.row_from[row]);
      hi = min(max(pos, prefix - 1), len - 1);
      if (a.slopes) slope = a.slopes[u.h * a.G + head] * kLog2e;
      see[0] = min(see[0], lo);
      see[1] = max(see[1], hi);
      see[2] = max(see[2], lo);
      see[3] = min(see[3], hi);
    }
    float off = 0.f;                           // a row with an infinity or a NaN gives NaN, and no other row does
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f[8];
      cvt8<BF16>(raw[i], f);
#pragma unroll
      for (int y = 0; y < 8; ++y) off += f[y] * 0.f;
      parts<NP>(f, q[i]);
    }
    if (!(sum_of_column(off) == 0.f))
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i][0] = __builtin_bit_cast(bf16x8, make_uint4(~0u, ~0u, ~0u, ~0u));
    clear();
  }
  // Products of N x 4 tokens to logits in powers of two, but for the factor that is returned, and less cap_out (not in kShapedFar);
  // at(j): the position of the first four of s[j]
  template <int N, class At>
  __device__ __forceinline__ float logits(const AttnArgs& a, f32x4 (&s)[N], At at) const {
    float scale = a.scale_log2;
    if constexpr (SHAPE == kPlain) return scale;
    if (a.cap_in != 0.f) {
      scale = 2.f * a.cap_out;
      if constexpr (SHAPE == kShaped) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)          // tanh x = 1 - 2 / (e^2x + 1)
            s[j][i] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(s[j][i] * a.cap_in));
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[j][i] = half_tanh(s[j][i] * a.cap_in);
      }
    }
    if (a.slopes) {
      const float far = (float)(at(0) - pos);  // (below 2^24: exact, and its sums)
      if (a.prefix_len) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[j][i] = __builtin_fmaf(s[j][i], scale, -slope * fabsf(far + (float)(at(j) - at(0) + i)));
      } else {                                 // what is seen lies before the row
        const float bias = slope * far;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[j][i] = __builtin_fmaf(s[j][i], scale, __builtin_fmaf(slope, (float)(at(j) - at(0) + i), bias));
      }
      scale = 1.f;
    }
    return scale;
  }
  // Hides what the column does not see, and tiles that are none
  template <int N, class At, class None>
  __device__ __forceinline__ void hide(f32x4 (&s)[N], At at, None none) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((int)none(j) | (at(j) + i < lo) | (at(j) + i > hi)) s[j][i] = -INFINITY;
  }
  // Logits, times `scale` > 0, to weights
  template <int N>
  __device__ __forceinline__ void soften(const f32x4 (&s)[N], float scale, float (&p)[4 * N]) {
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) mx = max3(max3(mx, s[j][0], s[j][1]), s[j][2], s[j][3]);
    mx *= scale;
    if (__any(mx > m - (kHead - kSlack))) {
      mx = max_of_column(mx);
      // (a column that does not need it stays, so that no row's result depends on its neighbours)
      const float to = mx > m - (kHead - kSlack) ? mx + kHead : m, down = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= down;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= down;
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * j + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][i], scale, -m));
        sum[i] += p[4 * j + i];
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // Another partial result's accumulators joined to these.  lane_of(i): who had o[i], col: its maximum and sum's place
  template <class Lane>
  __device__ __forceinline__ void join(const u64* part, int col, Lane lane_of) {
    const u64 ml = load_agent(part + 16 * kWave + col);
    u64 y[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i][0] = load_agent(part + i * 2 * kWave + lane_of(i));
      y[i][1] = load_agent(part + (i * 2 + 1) * kWave + lane_of(i));
    }
    const float l2 = as_f32((u32)(ml >> 32)), m2 = l2 == 0.f ? kLowest : as_f32((u32)ml);
    const float to = fmaxf(m, m2), f1 = __builtin_amdgcn_exp2f(m - to), f2 = l2 == 0.f ? 0.f : __builtin_amdgcn_exp2f(m2 - to);
    m = to;
    l = l * f1 + l2 * f2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f32x4 z = {as_f32((u32)y[i][0]), as_f32((u32)(y[i][0] >> 32)), as_f32((u32)y[i][1]), as_f32((u32)(y[i][1] >> 32))};
      o[i] = o[i] * f1 + z * f2;
    }
  }
};

__device__ __forceinline__ Seen seen_of(int (&see)[4]) {
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    see[0] = min(see[0], __shfl_xor(see[0], x, kWave));
    see[1] = max(see[1], __shfl_xor(see[1], x, kWave));
    see[2] = max(see[2], __shfl_xor(see[2], x, kWave));
    see[3] = min(see[3], __shfl_xor(see[3], x, kWave));
  }
  Seen s;
  s.first = __builtin_amdgcn_readfirstlane(see[0]) / kTile;
  s.behind = (__builtin_amdgcn_readfirstlane(see[1]) + kTile) / kTile;
  s.lo = __builtin_amdgcn_readfirstlane(see[2]);
  s.hi = __builtin_amdgcn_readfirstlane(see[3]);
  return s;
}

// N elements of a column's result over all tokens; the weights were taken times 2^-DOWN
template <bool BF16, int SHAPE, int DOWN, int N>
__device__ __forceinline__ void emit(const AttnArgs& a, const Unit& u, int r, int head, int d, const float (&v)[N], float m, float l) {
  const size_t at = (size_t)(u.row0 + r) * a.H * a.G + u.h * a.G + head;
  const float inv = l == 0.f ? 0.f : two_to(DOWN) / l;
  u32 w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = pack2<BF16>(l == 0.f ? 0.f : v[2 * i] * inv, l == 0.f ? 0.f : v[2 * i + 1] * inv);
  if constexpr (N == 8) *reinterpret_cast<uint4*>(a.out + at * kHeadDim + d) = make_uint4(w[0], w[1], w[2], w[3]);
  else *reinterpret_cast<uint2*>(a.out + at * kHeadDim + d) = make_uint2(w[0], w[1]);
  if (a.lse != nullptr && d == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l) + (SHAPE == kShapedFar ? 0.f : a.cap_out)) * kLn2;
}

// Tiles of a sequence's pages
struct Tiles {
  const AttnArgs& a;
  const Unit& u;
  const int tpp;
  __device__ __forceinline__ Tiles(const AttnArgs& a_, const Unit& u_) : a(a_), u(u_), tpp(a_.P / kTile) {}
  __device__ __forceinline__ int page_of(int t) const { return tpp == 1 ? t : (int)__umulhi(t, a.page_magic); }
  __device__ __forceinline__ int block(int t) const { return a.table[(size_t)u.seq * a.NP + page_of(t)]; }
  // Place of tile t, whose page has this block, in lines of 128 bytes; none behind t1 or of a block that is none
  __device__ __forceinline__ u32 line(int t, int t1, int b) const {
    const int sub = t - page_of(t) * tpp;
    return t < t1 && (unsigned)b < (unsigned)a.NB ? (((u32)b * a.H + u.h) * tpp + sub) * (kTileBytes / 128) : kNoTile;
  }
};
// The pool's first tile where there is none: what is read there is hidden
__device__ __forceinline__ const unsigned char* tile_at(const AttnArgs& a, u32 line) { return a.pages + (size_t)(line == kNoTile ? 0u : line) * 128; }

// ---- few rows

// A wave's 128 tokens at a time, keys and values of the next on their way.  Values' scales are one for 32 elements of a token, which the
// second product sums over: they go into the weights, so that each group of 32 columns of V has weights of its own, p * 2^e.  Where
// columns would be empty they repeat the rows (REP): each copy weighs the values of a fraction of the groups.  CG waves share tokens
// and have 16 columns each.
// One row a sequence is bound by the memory: 16 x 32768 tokens of 8 heads 101 to 105 us (5.5 TB/s), f16 107; 4 contexts of up to 1000 tokens
// 11.9 us by their chain of trips to memory.  More columns are bound by the vector unit's instructions, some 580 to 1100 for 128 tokens of a wave,
// which two waves a SIMD issue one each 4.5 cycles: 24 ragged contexts with up to 3 rows of 7 x 4 heads, f16, capped and sloped, 116 us (2.5
// TB/s), 64 for one row in bf16.  (With one part of weights, 64 tokens at a time and three waves a SIMD: 117 us for 99, as each step has as
// much around it.)
// What a lane would not need all the time lies in LDS, its wave's scales of values and, where registers are short, its queries: spilled
// ones came back behind the loads on their way, and the wait for them was one for all of those (the drafts 133 us, with the queries
// alone in LDS 126).
template <bool BF16, int SHAPE, int REP, int CG>
struct Wave {
  static constexpr int NP = Columns<BF16, SHAPE, kFewHead>::NP;
  static constexpr int kCols = 16 / REP;       // columns that differ
  static constexpr int kGroups = 4 / REP;      // of V's groups of 32 columns, those that a lane weighs
  static_assert(CG == 1 || REP == 1, "");
  // (bf16 with a cap, 16 x 32768 tokens 110 us; without one, two groups of columns spill 2 registers and four groups 10 where they hold them)
  static constexpr bool kPutBy = !BF16 || SHAPE != kPlain || CG > 1;
  Columns<BF16, SHAPE, kFewHead> x;
  Seen seen;

  const AttnArgs& a;
  const int lane, c, n, cg;                    // cg: which columns of the unit are the wave's
  Unit u;

  __device__ __forceinline__ Wave(const AttnArgs& a_)
      : a(a_), lane(threadIdx.x % kWave), c((threadIdx.x % kWave) >> 4), n(threadIdx.x & 15),
        cg(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave) % CG) {}

  // Queries, where a step takes them from LDS
  static __device__ __forceinline__ uint4* put_by() {
    __shared__ uint4 at[kPutBy ? 4 * NP * kAttnThreads : 1];
    return at + threadIdx.x;
  }
  // Row of the unit and head of the group of column col
  __device__ __forceinline__ bool column(int col, int& r, int& head) const {
    r = col / a.G;
    head = col - r * a.G;
    return r < u.rows && r < a.R;
  }
  // whether this lane's accumulators of 16 columns of V are of the weights that were made for them
  __device__ __forceinline__ bool has(int i) const { return REP == 1 || (i >> 1) % REP == n / kCols; }
  // Lane that has column col's accumulators of 16 columns of V
  __device__ __forceinline__ int lane_of(int i, int col, int quarter) const {
    return quarter * 16 + (REP == 1 ? col : col % kCols + (i >> 1) % REP * kCols);
  }

  __device__ __forceinline__ void begin(const Unit& unit) {
    u = unit;
    const int len = min(max(a.kv_len[u.seq], 0), a.NP * a.P);
    const int prefix = a.prefix_len ? min(max(a.prefix_len[u.seq], 0), len) : 0;
    int see[4] = {0x7fffffff, -1, 0, 0x7fffffff}, r, head;
    const bool ok = column(cg * 16 + n % kCols, r, head);
    x.begin(a, u, ok, r, head, len, prefix, see);
    seen = seen_of(see);
    if constexpr (kPutBy)
#pragma unroll
      for (int i = 0; i < 4 * NP; ++i) put_by()[i * kAttnThreads] = __builtin_bit_cast(uint4, x.q[i / NP][i % NP]);
  }

  // ---- what is on its way

  i32x4 k[8], v[8];
  u32 ks[2];
  u64 vs;                                      // of the 32 tokens that the lanes (c, *) have, scales of 8 values, of group n % 8 / 2
  u32 line, line_next;                         // of the step's tile lane % 8
  int block_next;                              // of the step after that

  __device__ __forceinline__ const unsigned char* tile(u32 lines, int i) const { return tile_at(a, __shfl(lines, i, kWave)); }
  __device__ __forceinline__ void load_keys(u32 lines) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const unsigned char* at = tile(lines, 2 * (n >> 2) + half) + (n & 3) * 64 + c * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) k[half * 4 + j] = load_codes<CG == 1>(at + j * 256);
      ks[half] = *reinterpret_cast<const u32*>(at - (n & 3) * 60 + kKeyScales);
    }
  }
  __device__ __forceinline__ void load_values(u32 lines) {
    const unsigned char *at0 = tile(lines, 2 * c), *at1 = tile(lines, 2 * c + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = load_codes<CG == 1>(at0 + kValues + n * 16 + i * 256);
      v[2 * i + 1] = load_codes<CG == 1>(at1 + kValues + n * 16 + i * 256);
    }
    vs = *reinterpret_cast<const u64*>((n < 8 ? at0 : at1) + kValueScales + (n & 7) * 8);
  }
  // In LDS, for each c: scales of two tiles, four groups and 16 tokens
  static __device__ __forceinline__ u64* scales_of(int wave) {
    __shared__ __align__(16) u64 at[kAttnThreads];
    return at + wave * kWave;
  }

  // ---- the step of tiles [t0, t0 + 8)

  // Row r of the products of tile j is token 32 (r / 4) + 4 j + r % 4 of the step, so that lane (c, n) gets tokens 32 c + 0..31 of column n
  __device__ __forceinline__ void scores(f32x4 (&s)[8]) {
    bf16x8 q[4][NP];
    int none = 0;
    asm volatile("" : "+v"(none));             // (taken anew each time)
#pragma unroll
    for (int i = 0; i < 4 * NP; ++i) q[i / NP][i % NP] = kPutBy ? __builtin_bit_cast(bf16x8, put_by()[i * kAttnThreads + none]) : x.q[i / NP][i % NP];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float scale = two_to((int)byte_of(ks[j / 4], j % 4) - kBias);
      s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 A = widen(k[j][i], scale);
#pragma unroll
        for (int p = 0; p < NP; ++p) s[j] = mfma32(A, q[i][p], s[j]);
      }
    }
  }
  // What the tokens add to 32 columns of V (REP > 1: to REP groups of them, of which one has this lane's weights).  p * 2^(e - 126): a
  // bf16's bits less 126 - e in its exponent, which are those of a smaller number, and 0 where there would be none; p is up to 2^98.
  template <int X>
  __device__ __forceinline__ void weigh(const u16x2 (&p)[4][kWeightParts][4]) {
    const u32 times = 0x10001u * (u32)(0x10000 - 128), most = 0x10001u * ((kBias + kFewDown) << 7);
    const u64* from = scales_of(threadIdx.x / kWave) + c * 16 + (X * REP + (REP > 1 ? n / kCols : 0)) * 2;
    const i32x4 scales[2] = {*reinterpret_cast<const i32x4*>(from), *reinterpret_cast<const i32x4*>(from + 8)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {              // eight of the lane's tokens
      bf16x8 B[kWeightParts];
      u16x2 w[kWeightParts][4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const u32 bytes = __builtin_amdgcn_perm(0, (u32)scales[i >> 1][(i & 1) * 2 + (y >> 1)], y & 1 ? 0x0c030c02 : 0x0c010c00);
        const u16x2 down = mad_pair(bytes, times, most);
#pragma unroll
        for (int z = 0; z < kWeightParts; ++z) w[z][y] = __builtin_elementwise_sub_sat(p[i][z][y], down);
      }
#pragma unroll
      for (int z = 0; z < kWeightParts; ++z) B[z] = __builtin_bit_cast(bf16x8, w[z]);
#pragma unroll
      for (int z = 0; z < 2 * REP; ++z) {
        const int d = X * 2 * REP + z;         // 16 columns
        const bf16x8 A = widen(v[d / 2 * 2 + (i >> 1)][d % 2 * 2 + (i & 1)], 1.f);
#pragma unroll
        for (int y = 0; y < kWeightParts; ++y) x.o[d] = mfma32(A, B[y], x.o[d]);
      }
    }
  }

  // Tiles [from, to) of the unit.  Keys of the next step are asked for when those of this one have been taken, values likewise;
  // the blocks of the tiles two steps ahead.  (Behind the last step too, where there is no tile: a wait counts the loads behind
  // what it waits for, and has to find as many whichever way the code came.)
  __device__ __forceinline__ void sweep(int from, int to) {
    if (from < to) {
      const Tiles tiles(a, u);
      const int t8 = lane & 7, last = to - 1;
      line = tiles.line(from + t8, to, tiles.block(min(from + t8, last)));
      block_next = tiles.block(min(from + kStep + t8, last));
      load_keys(line);
      load_values(line);
      for (int t = from; t < to; t += kStep) {
        f32x4 s[8];
        scores(s);
        __builtin_amdgcn_sched_barrier(0);
        line_next = tiles.line(t + kStep + t8, to, block_next);
        block_next = tiles.block(min(t + 2 * kStep + t8, last));
        load_keys(line_next);
        __builtin_amdgcn_sched_barrier(0);
        const int base = t * kTile;
        auto at = [&](int j) { return base + c * 32 + j * 4; };
        const float scale = x.logits(a, s, at);
        if (base < seen.lo || base + kStep * kTile - 1 > seen.hi || __any(line == kNoTile)) {
          const bool none[2] = {__shfl(line, 2 * c, kWave) == kNoTile, __shfl(line, 2 * c + 1, kWave) == kNoTile};
          x.hide(s, at, [&](int j) { return none[j >> 2]; });
        }
        float p[32];
        x.soften(s, scale, p);
        u16x2 w[4][kWeightParts][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) weights(p + 8 * i, w[i]);
        scales_of(threadIdx.x / kWave)[lane] = vs;
        each_of<kGroups>([&](auto g) { weigh<decltype(g)::value>(w); });
        __builtin_amdgcn_sched_barrier(0);
        line = line_next;
        load_values(line);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    x.l = sum_of_column(x.l);                  // a column's four lanes have a quarter of its sum each
  }

  // Partial results of other workgroups, as this launch's lanes have them: accumulators [i][half][lane] in pairs, then (maximum, sum) [n]
  __device__ __forceinline__ u64* part_of(int slot, int group) const { return a.part + ((size_t)slot * CG + group) * kPartWords; }
};

struct AttnLds {
  float ml[kAttnWaves][16][2];
  __align__(16) float o[kAttnWaves][16][kColFloats];
  int last;
};

// The results of the waves that share columns as one: with to_slot < 0 to the output, else there
template <bool BF16, int SHAPE, int REP, int CG>
__device__ __forceinline__ void merge_waves(const AttnArgs& a, const Wave<BF16, SHAPE, REP, CG>& w, AttnLds& lds, int to_slot) {
  typedef Wave<BF16, SHAPE, REP, CG> W;
  const int tid = threadIdx.x, wave = tid / kWave;
  __syncthreads();                             // (what was there has been read)
  if (w.c == 0) {
    lds.ml[wave][w.n][0] = w.x.l == 0.f ? kLowest : w.x.m;
    lds.ml[wave][w.n][1] = w.x.l;
  }
  __syncthreads();
  float M = kLowest;
#pragma unroll
  for (int i = 0; i < kAttnWaves; i += CG) M = fmaxf(M, lds.ml[i + w.cg][w.n][0]);
  const float f = w.x.l == 0.f ? 0.f : __builtin_amdgcn_exp2f(w.x.m - M);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (w.has(i)) *reinterpret_cast<f32x4*>(&lds.o[wave][w.n % W::kCols][i * 16 + w.c * 4]) = w.x.o[i] * f;
  __syncthreads();
  const int n = tid >> 4, d = (tid & 15) * 8;  // a column and eight of its elements
#pragma unroll
  for (int g = 0; g < CG; ++g) {
    int r, head;
    if (n < W::kCols && w.column(g * 16 + n, r, head)) {
      float top = kLowest, L = 0.f, v[8];
#pragma unroll
      for (int i = g; i < kAttnWaves; i += CG) top = fmaxf(top, lds.ml[i][n][0]);
#pragma unroll
      for (int i = g; i < kAttnWaves; i += CG) {
        const float l = lds.ml[i][n][1];
        if (l != 0.f) L += l * __builtin_amdgcn_exp2f(lds.ml[i][n][0] - top);
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        v[y] = 0.f;
#pragma unroll
        for (int i = g; i < kAttnWaves; i += CG) v[y] += lds.o[i][n][d + y];
      }
      if (to_slot < 0) emit<BF16, SHAPE, kFewDown>(a, w.u, r, head, d, v, top, L);
      else {
        u64* part = w.part_of(to_slot, g);
        const int i = d / 16;
#pragma unroll
        for (int y = 0; y < 4; ++y)
          store_agent(part + (i * 2 + (y & 1)) * kWave + w.lane_of(i, n, d % 16 / 4 + (y >> 1)), pack_floats(v[2 * y], v[2 * y + 1]));
        if (d == 0) store_agent(part + 16 * kWave + n, pack_floats(top, L));
      }
    }
  }
}

// Tiles [t0, t1) of a unit: by all waves, or, if they are one step (`step`), by those of turn `solo` alone.  Its result goes to the output if it is
// all of the unit (count == 1), else to slot `mine` of the partial results, which the last of the `count` pieces to arrive
// joins, in their order; slot(i) is the i-th one's number.
template <bool BF16, int SHAPE, int REP, int CG, class Slot>
__device__ __forceinline__ void piece(const AttnArgs& a, Wave<BF16, SHAPE, REP, CG>& w, AttnLds& lds, const Unit& u, int t0, int t1,
                                      bool step, int solo, int count, int mine, int ticket, Slot slot) {
  constexpr int kShares = kAttnWaves / CG;
  const int share = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) / CG;
  // (pieces of one unit are joined in one way, whichever comes last: the sums' order is fixed)
  const bool alone = count == 1 && (step || kShares == 1);
  if (alone && share != solo % kShares) return;
  w.begin(u);
  t0 = max(t0, w.seen.first);
  t1 = max(min(t1, w.seen.behind), t0);
  if (!alone) {
    const int per = ((t1 - t0 + kStep - 1) / kStep + kShares - 1) / kShares * kStep;
    t0 = min(t0 + share * per, t1);
    t1 = min(t0 + per, t1);
  }
  w.sweep(t0, t1);
  if (alone) {
    int r, head;
    if (!w.column(w.cg * 16 + w.n % w.kCols, r, head)) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (!w.has(i)) continue;
      const float v[4] = {w.x.o[i][0], w.x.o[i][1], w.x.o[i][2], w.x.o[i][3]};
      emit<BF16, SHAPE, kFewDown>(a, u, r, head, i * 16 + w.c * 4, v, w.x.m, w.x.l);
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
  w.x.clear();
  for (int i = share; i < count; i += kShares)
    w.x.join(w.part_of(slot(i), w.cg), w.n % w.kCols, [&](int y) { return w.lane_of(y, w.n, w.c); });
  merge_waves(a, w, lds, -1);
}

// What a window leaves of a unit: tiles at most, and the first one
__device__ __forceinline__ bool windowed(const AttnArgs& a) { return a.window > 0 && a.prefix_len == nullptr; }
__device__ __forceinline__ int most_tiles(const AttnArgs& a) {
  return windowed(a) ? (int)min(((long long)a.window + a.R + 2 * kTile - 3) / kTile, (long long)q8::kAllTiles) : q8::kAllTiles;
}
// Where its tiles are counted from: a unit's first piece has what lies before that too
__device__ __forceinline__ int first_tile(const AttnArgs& a, const Unit& u) {
  return max(u.lead, windowed(a) ? max(u.pos0 - a.window + 1, 0) / kTile : 0);
}
// Tiles of a sequence that its first row does not see, and no other row as a rule
__device__ __forceinline__ auto lead_of(const AttnArgs& a) {
  return [&a](int row0) { return a.row_from && row0 < a.T ? max(a.row_from[row0], 0) / kTile : 0; };
}

template <bool BF16, int SHAPE, int REP, int CG>
__global__ __launch_bounds__(kAttnThreads, 2) void q4_attn_kernel(AttnArgs a) {
  __shared__ AttnLds lds;
  Wave<BF16, SHAPE, REP, CG> w(a);
  int solo = 0;
  deal<kAttnThreads, kLeastTiles, kPieceTiles, kFewPad>(a, false, most_tiles(a), lead_of(a), [&](const Unit& u, int t0, int t1, int f, int count,
                                                                                                  int mine, auto slot) {
    const int first = first_tile(a, u);
    piece(a, w, lds, u, t0 > 0 ? first + t0 : 0, first + t1, t1 - t0 <= kStep, solo, count, mine, f, slot);
    ++solo;
  });
}

// ---- many rows

// Each wave has its own kRowGroups * 16 columns, and the workgroup's WAVES go through the tokens together, 64 at a time: waves fetch a
// tile each, widen it and put it into LDS in operand order, while the 64 before it are taken; so a code is widened once for all
// of them.  Values take their scales there.  Of eight waves four have the keys and four the values.
// Bound by issue and by phases that all waves are in at once: about 410 vector instructions, 96 products (a third of them for the
// second part of the weights) and 33 trips to LDS a wave and stage, two waves a SIMD, vector unit and matrix cores busy 55 % and 40 to 45 %
// of the time.  2 x 2048 rows of 32/8 heads behind 6144 tokens 668 us (720 TFLOP/s without the second part's), in documents of 5000 tokens
// 245 to 260 (580), 2 x 4096 rows from the start 440 (630); the documents in f16 309, with a cap 296, with slopes too 342, f16 374.  (With
// one part of weights 32 x 32 products took 229 us for 210, as only two chains of them go at a time.)
constexpr int kRowGroups = 2;
constexpr int kStageTiles = 4;
template <int WAVES>
struct RowsLds {
  uint4 k[2][kStageTiles][4][kWave];           // [stage][tile][8 elements of 32][lane]
  uint4 v[2][kStageTiles / 2][8][kWave];       // [stage][pair of tiles][16 elements][lane]
  u32 line[2][kStageTiles];
  int first[WAVES], behind[WAVES];
};

template <bool BF16, int SHAPE, int WAVES>
__global__ __launch_bounds__(WAVES* kWave, 2) void q4_attn_rows_kernel(AttnArgs a) {
  constexpr int NQ = kRowGroups, NP = Columns<BF16, SHAPE, kRowsHead>::NP;
  __shared__ RowsLds<WAVES> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, c = lane >> 4, n = lane & 15;
  const int rows = a.R / WAVES;                // of a wave
  const int tile = wave % kStageTiles;         // of a stage, the one that this wave fetches
  const bool keys = wave < kStageTiles, values = WAVES == kStageTiles || !keys;
  Columns<BF16, SHAPE, kRowsHead> x[NQ];
  const bool grow = !windowed(a) && a.prefix_len == nullptr;
  deal<WAVES * kWave, kLeastTiles, 0, kRowsPad>(a, grow, most_tiles(a), lead_of(a), [&](const Unit& whole, int t0, int t1, int f, int count,
                                                                                         int mine, auto slot) {
    Unit u = whole;                            // this wave's rows
    u.row0 += wave * rows;
    u.pos0 += wave * rows;
    u.rows = min(max(whole.rows - wave * rows, 0), rows);
    const Tiles tiles(a, whole);
    const int len = min(max(a.kv_len[u.seq], 0), a.NP * a.P);
    const int prefix = a.prefix_len ? min(max(a.prefix_len[u.seq], 0), len) : 0;
    int see[4] = {0x7fffffff, -1, 0, 0x7fffffff};
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      const int col = g * 16 + n, r = col / a.G;
      x[g].begin(a, u, r < u.rows, r, col - r * a.G, len, prefix, see);
    }
    const Seen seen = seen_of(see);
    __syncthreads();                           // (the last piece's stages have been read)
    if (lane == 0) { lds.first[wave] = seen.first; lds.behind[wave] = seen.behind; }
    __syncthreads();
    const int first = first_tile(a, whole);
    int from = lds.first[0], to = lds.behind[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) { from = min(from, lds.first[i]); to = max(to, lds.behind[i]); }
    from = __builtin_amdgcn_readfirstlane(max(t0 > 0 ? first + t0 : 0, from));
    to = __builtin_amdgcn_readfirstlane(min(first + t1, to));

    i32x4 kc = {}, vc = {}, vsc = {};          // this wave's tile on its way: codes of keys and values, scales of values
    u32 ksc = 0, line = kNoTile;
    int block = -1;
    auto fetch = [&](int t) {                  // tile t, whose block is at hand, and the block of the one after it
      line = tiles.line(t, to, block);
      block = tiles.block(min(t + kStageTiles, to - 1));
      const unsigned char* at = tile_at(a, line);
      if (keys) {
        kc = load_scales(at + n * 64 + c * 16);
        ksc = at[kKeyScales + c * 16 + (n & 3) * 4 + (n >> 2)];
      }
      if (values) {
        vc = load_scales(at + kValues + lane * 16);
        vsc = load_scales(at + kValueScales + c * 16);
      }
    };
    auto put = [&](int s) {
      if (keys) {
        const float scale = two_to((int)ksc - kBias);
#pragma unroll
        for (int i = 0; i < 4; ++i) lds.k[s][tile][i][lane] = __builtin_bit_cast(uint4, widen(kc[i], scale));
        if (lane == 0) lds.line[s][tile] = line;
      }
      if (!values) return;
      // lane l has elements 32 (l / 16) + l % 16 and 16 more, 16 tokens each: two tokens of a byte, a scale each
      u64* to_v = reinterpret_cast<u64*>(&lds.v[s][tile >> 1][2 * c][n]) + (tile & 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {            // tokens 4 i + 0..3, which are lane (i, n)'s
        float e[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) e[y] = two_to((int)min(byte_of(vsc[i], y), (u32)(kExpMax + kBias)) - kBias);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const u32 w = (u32)vc[half * 2 + (i >> 1)];
          const u32 first = (i & 1) ? pair<2>(w, e[0], e[1]) : pair<0>(w, e[0], e[1]);
          const u32 second = (i & 1) ? pair<3>(w, e[2], e[3]) : pair<1>(w, e[2], e[3]);
          to_v[(half * kWave + i * 16) * 2] = (u64)second << 32 | first;
        }
      }
    };
    if (from < to) {
      block = tiles.block(min(from + tile, to - 1));
      fetch(from + tile);
      put(0);
      __syncthreads();
      int stage = 0;
      for (int t = from; t < to; t += kStageTiles, stage ^= 1) {
        fetch(t + kStageTiles + tile);
        if (t < seen.behind && t + kStageTiles > seen.first) {
          // operands are asked for four at a time, while the four before them are taken: keys of two tiles, two of their four
          // parts each, then values of a pair of tiles, four of their eight
          uint4 b[2][4];
          auto ask = [&](int i) {
#pragma unroll
            for (int y = 0; y < 4; ++y)
              b[i & 1][y] = i < 4 ? lds.k[stage][i / 2 * 2 + (y & 1)][i % 2 * 2 + (y >> 1)][lane] : lds.v[stage][i / 2 - 2][i % 2 * 4 + y][lane];
            __builtin_amdgcn_sched_barrier(0);
          };
          ask(0);
          f32x4 s[NQ][4];
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ask(i + 1);
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int g = 0; g < NQ; ++g)
                  s[g][i / 2 * 2 + (y & 1)] = mfma32(__builtin_bit_cast(bf16x8, b[i & 1][y]), x[g].q[i % 2 * 2 + (y >> 1)][p],
                                                    i % 2 == 0 && y < 2 && p == 0 ? zero : s[g][i / 2 * 2 + (y & 1)]);
          }
          const int base = t * kTile;
          auto at = [&](int j) { return base + j * kTile + c * 4; };
          u32 gone = 0;                        // bit j: tile j is none
#pragma unroll
          for (int j = 0; j < kStageTiles; ++j) gone |= lds.line[stage][j] == kNoTile ? 1u << j : 0u;
          gone = __builtin_amdgcn_readfirstlane(gone);
          const bool hide = base < seen.lo || base + kStageTiles * kTile - 1 > seen.hi || gone;
          bf16x8 B[NQ][2][kWeightParts];
#pragma unroll
          for (int g = 0; g < NQ; ++g) {
            const float scale = x[g].logits(a, s[g], at);
            if (hide) x[g].hide(s[g], at, [&](int j) { return (gone >> j & 1) != 0; });
            float p[16];
            x[g].soften(s[g], scale, p);
            parts<kWeightParts>(p, B[g][0]);
            parts<kWeightParts>(p + 8, B[g][1]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i < 3) ask(i + 5);
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int p = 0; p < kWeightParts; ++p)
#pragma unroll
                for (int g = 0; g < NQ; ++g)
                  x[g].o[i % 2 * 4 + y] = mfma32(__builtin_bit_cast(bf16x8, b[i & 1][y]), B[g][i / 2][p], x[g].o[i % 2 * 4 + y]);
          }
        }
        if (t + kStageTiles < to) {
          put(stage ^ 1);
          __syncthreads();
        }
      }
    }
    bool last = true;
#pragma unroll
    for (int g = 0; g < NQ; ++g) x[g].l = sum_of_column(x[g].l);
    if (count > 1) {
      auto part_of = [&](int i, int g) { return a.part + (((size_t)i * WAVES + wave) * NQ + g) * kPartWords; };
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        u64* part = part_of(mine, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          store_agent(part + i * 2 * kWave + lane, pack_floats(x[g].o[i][0], x[g].o[i][1]));
          store_agent(part + (i * 2 + 1) * kWave + lane, pack_floats(x[g].o[i][2], x[g].o[i][3]));
        }
        if (c == 0) store_agent(part + 16 * kWave + n, pack_floats(x[g].m, x[g].l));
      }
      wave_drain_memory();                     // (written through and drained before the ticket, and read past the caches)
      int before = 0;
      if (lane == 0) before = __hip_atomic_fetch_add(a.ticket + f * WAVES + wave, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __builtin_amdgcn_readfirstlane(before) == count - 1;
      if (last) {
        if (lane == 0) store_agent(a.ticket + f * WAVES + wave, 0);
#pragma unroll
        for (int g = 0; g < NQ; ++g) x[g].clear();
        for (int i = 0; i < count; ++i)
#pragma unroll
          for (int g = 0; g < NQ; ++g) x[g].join(part_of(slot(i), g), n, [&](int) { return lane; });
      }
    }
    if (last)
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        const int col = g * 16 + n, r = col / a.G;
        if (r >= u.rows) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v[4] = {x[g].o[i][0], x[g].o[i][1], x[g].o[i][2], x[g].o[i][3]};
          emit<BF16, SHAPE, 0>(a, u, r, col - r * a.G, i * 16 + c * 4, v, x[g].m, x[g].l);
        }
      }
  });
}

// How the columns that the rows of a sequence take, on the average, are laid out: copies of them in 16, or groups of 16 (0: workgroups
// of 4 or 8 waves with rows of their own).  us: 30 x up to 3000 tokens, 4 columns: four copies 21.7, one 22.1.  16 x 6000 tokens of 8
// heads, 64 columns: four groups 85, 4 waves with rows 103; 96: 125, 107; 128: 130, 112, and 8 waves with rows 120; 160: 4 waves 171, 8
// waves 162; 252: 181, 183.  All sequences of a step have one layout, which is right for those that are alike: 63 single tokens
// behind 32768 take 389 us and 2048 rows behind 6144 368, but a step of all of them 3267, its single tokens in waves with rows (with
// 512 rows 114, and 1101 together, those rows in units of 16 columns).
struct Shape { int copies, groups, waves; };
static Shape shape_of(int T, int B, int G) {
  const int64_t want = (int64_t)((T + B - 1) / B) * G;
  return {want <= 4 ? 4 : want <= 8 ? 2 : 1, want <= 16 ? 1 : want <= 32 ? 2 : want <= 64 ? 4 : 0, want <= 128 ? 4 : 8};
}

}  // namespace q4
}  // namespace kvd

extern "C" int64_t kvd_q4_workspace_bytes(const kvd_q4_cache* c, const kvd_q8_rows* r) {
  using namespace kvd::q4;
  if (int e = check_cache(c, r)) return e;
  static_assert(kAttnGroups * kAttnWaves * 4 <= kvd::q8::kTicketBytes, "a ticket for each wave of each workgroup");
  const Shape shape = shape_of(r->n_rows, r->n_seqs, c->n_q_heads / c->n_kv_heads);
  // (with 8 waves half as many workgroups)
  return kvd::q8::kTicketBytes + (int64_t)kAttnGroups * 2 * 8 * kPartWords * (shape.groups ? shape.groups : kAttnWaves * kRowGroups);
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
  a.scale_log2 = fminf(fmaxf((c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e, 0x1p-126f), 0x1.fffffep127f);
  if (f) {
    if (!(f->softcap >= 0.f) || f->softcap > 0x1p96f) return KVD_ERR_ARG;
    if (f->window < 0) return KVD_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(f->slopes) | reinterpret_cast<uintptr_t>(f->row_from) | reinterpret_cast<uintptr_t>(f->prefix_len)) & 3)
      return KVD_ERR_ARG;
    if (f->softcap > 0.f) {
      a.cap_in = 2.f * a.scale_log2 / f->softcap;
      a.cap_out = f->softcap * kLog2e;
      if (!(a.cap_in >= 0x1p-126f) || isinf(a.cap_in)) return KVD_ERR_ARG;
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
  const int tpp = a.P / kTile;
  a.page_magic = (kvd::u32)(((1ull << 32) + tpp - 1) / tpp);
  const Shape shape = shape_of(a.T, a.B, a.G);
  a.R = shape.groups ? 16 * shape.groups / shape.copies / a.G : 16 * kRowGroups / a.G * shape.waves;
  a.W = shape.groups || shape.waves == kAttnWaves ? kAttnGroups : kAttnGroups / 2;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto go = [&](auto kernel, int waves = kAttnWaves) { hipLaunchKernelGGL(kernel, dim3(a.W), dim3(waves * kvd::kWave), 0, s, a); };
  auto typed = [&](auto bf16, auto shape_of_scores) {
    constexpr bool B = decltype(bf16)::value;
    constexpr int S = decltype(shape_of_scores)::value;
    if (shape.copies == 4) go(q4_attn_kernel<B, S, 4, 1>);
    else if (shape.copies == 2) go(q4_attn_kernel<B, S, 2, 1>);
    else if (shape.groups == 1) go(q4_attn_kernel<B, S, 1, 1>);
    else if (shape.groups == 2) go(q4_attn_kernel<B, S, 1, 2>);
    else if (shape.groups == 4) go(q4_attn_kernel<B, S, 1, 4>);
    else if (shape.waves == 4) go(q4_attn_rows_kernel<B, S, 4>);
    else go(q4_attn_rows_kernel<B, S, 8>, 8);
  };
  auto shaped = [&](auto bf16) {
    if (a.cap_in == 0.f && a.slopes == nullptr) typed(bf16, std::integral_constant<int, kPlain>{});
    else if (a.cap_in == 0.f || f->softcap <= kNearCap) typed(bf16, std::integral_constant<int, kShaped>{});
    else typed(bf16, std::integral_constant<int, kShapedFar>{});
  };
  if (c->kv_dtype == KVD_BF16) shaped(std::true_type{}); else shaped(std::false_type{});
  return launched();
}
