// Attention of a step's rows over the pages of the 8-bit cache.
//
// S^T = K Q^T and O^T += V^T P^T on the matrix cores, 32 tokens at a time: a result's columns are query rows (a row of the
// step and a head of the group), and the softmaxed S^T of a lane is, register for register, its operand of the second
// product.  Tiles come from memory in operand order, 16 bytes a lane and load; codes become 16-bit numbers in registers, which
// holds every e4m3 value exactly.  The keys' scale goes into the logits, the values' into the conversion.
//
// One pass with a running reference m and sum l of a column: p = 2^(x - m).  m is kHead above the largest logit when it is set, and
// is raised only when a logit passes that by more than kSlack, so that the accumulators are rarely touched; p then stays below
// 2^(kSlack - kHead), and nothing is lost, as all of this is floating point.
//
// Nothing is infinite on the way either.  The largest value, 448 * 2^120, is beyond fp32; one that became an infinity would make NaN of
// every hidden weight of 0 too.  Values are taken times 2^-kValueDown, which leaves the least, 2^-105, a normal number; weights
// are below 2^-4, so that the sum of 2^24 tokens is below 2^(24 - 4 + 129 - 21) = 2^128.  Keys that are widened with their scale
// are taken times 2^-kKeyDown.
//
// Weights and values go to the second product in bf16, which has the range for any scale of a page: no page's scale, seen or
// hidden, costs another page's tokens anything.  (f16 has not: weights relative to the largest scale of a wave's pages lost
// all their bits where values were 2^30 apart.)  The weights' bits: DUP (one row of up to 8 heads): the 16 columns hold each head
// twice, and the second copy takes what rounding P to bf16 left of it: P is then 16 bits long at the price of nothing, as the
// columns would be empty.  TWO: a product more for that rest, which costs 2 % where a few rows wait for the memory.  Many rows of bf16
// do without it: P is rounded to bf16 there, by 2^-8 of each weight at most, like their output (530 us for 670 with it at 2 x 2048
// rows of 32/8 heads behind 6144 tokens; f16, whose outputs would show it, has it: 700).
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / kWave;
constexpr int kAttnGroups = 512;               // workgroups of the dense form: two for each CU
constexpr int kXcds = 8;                       // divides kAttnGroups
constexpr int kLeastTiles = 16;                // tiles of a workgroup at least
constexpr int kCoopTiles = 8;                  // from so many tiles on a unit is shared by the workgroup's waves
constexpr int kColFloats = kHeadDim + 4;       // a column in LDS
// 8-byte words of a wave's partial result: accumulators, then a maximum and a sum a column
__host__ __device__ constexpr size_t part_words(int groups) { return (size_t)groups * (16 * kWave + 16); }
constexpr float kLowest = -3.0e38f, kSlack = 8.f, kHead = 12.f;
constexpr int kValueDown = 21, kKeyDown = 2;
constexpr int kNowhere = 1 << 30;              // position of a tile that no row sees
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnArgs {
  const uint16_t* q;
  long long q_stride;
  const int32_t *table, *kv_len, *row_start, *row_seq, *row_pos, *sel;
  const unsigned char* pages;
  const int8_t* exps;
  uint16_t* out;
  float* lse;
  u64* part;
  int32_t* ticket;
  int B, NP, T, H, G, P, NB, k, R, W, S;       // R rows of a unit, W workgroups (dense), S splits of a unit (selected)
  float scale_log2;
};

// What the rows of one unit (up to R rows of a sequence, one head) have in common
struct Unit {
  int row0, rows, h, seq, pos0, entries;       // pos0: position of row0; entries: pages (or selected pages)
};

template <bool BF16> struct Op { typedef bf16x8 type; };
template <> struct Op<false> { typedef f16x8 type; };

template <bool BF16>
__device__ __forceinline__ f32x4 mfma32(typename Op<BF16>::type a, typename Op<BF16>::type b, f32x4 c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// Eight codes to an operand, times 2^e where scale is that
template <bool BF16>
__device__ __forceinline__ typename Op<BF16>::type widen(u32 lo, u32 hi, float s_lo, float s_hi) {
  u32 w[4];
  if constexpr (BF16) {
    w[0] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, false));
    w[1] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, true));
    w[2] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, false));
    w[3] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, true));
  } else {
    w[0] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, s_lo, false));
    w[1] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, s_lo, true));
    w[2] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, s_hi, false));
    w[3] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, s_hi, true));
  }
  return __builtin_bit_cast(typename Op<BF16>::type, make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ u32 word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

__device__ __forceinline__ u64 pack_floats(float a, float b) { return (u64)as_u32(b) << 32 | as_u32(a); }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// Two tiles on their way
struct Pair {
  uint4 k[2][2], v[2][2];
  int tok[2], ek[2], ev[2];
};

template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL>
struct Wave {
  static constexpr int kParts = TWO ? 2 : 1;   // operands of P
  f32x4 o[NQ][8];
  float m[NQ], l[NQ];
  typename Op<BF16>::type q[NQ][4];
  int lim[NQ];                                 // last position that the lane's column sees

  const AttnArgs& a;
  const int lane, c, n;
  Unit u;
  // the 64 page entries at hand: block and exponents of entry e0 + lane
  int e0, e, sub, t, t1, blk, ex, pg;

  __device__ __forceinline__ Wave(const AttnArgs& a_) : a(a_), lane(threadIdx.x % kWave), c((threadIdx.x % kWave) >> 4), n(threadIdx.x & 15) {}

  // Row of the unit and head of the group of column n + 16 g
  __device__ __forceinline__ void column(int g, int& r, int& head) const {
    if (DUP) { r = 0; head = n & 7; }
    else { const int col = n + 16 * g; r = col / a.G; head = col - r * a.G; }
  }
  __device__ __forceinline__ bool real(int r, int head) const { return head < a.G && r < u.rows; }

  __device__ __forceinline__ void begin(const Unit& unit) {
    u = unit;
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      int r, head;
      column(g, r, head);
      const bool ok = real(r, head);
      lim[g] = ok ? u.pos0 + r : -1;
      const uint16_t* src = a.q + (long long)(u.row0 + r) * a.q_stride + (u.h * a.G + head) * kHeadDim + c * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (ok) x = *reinterpret_cast<const uint4*>(src + j * 32);
        q[g][j] = __builtin_bit_cast(typename Op<BF16>::type, x);
      }
      m[g] = kLowest;
      l[g] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  __device__ __forceinline__ void fetch_entries() {
    const int i = e0 + lane;
    blk = -1;
    pg = 0;
    ex = 0;
    if (i < u.entries) {
      pg = SEL ? a.sel[((size_t)u.row0 * a.H + u.h) * a.k + i] : i;
      if ((unsigned)pg < (unsigned)a.NP) blk = a.table[(size_t)u.seq * a.NP + pg];
      if ((unsigned)blk >= (unsigned)a.NB) blk = -1;
      if (blk >= 0) ex = *reinterpret_cast<const int16_t*>(a.exps + ((size_t)blk * a.H + u.h) * 2);
    }
  }
  __device__ __forceinline__ void load(Pair& p) {
    const int tpp = a.P / kTile;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int b = -1;
      if (t < t1) {
        if (e - e0 == kWave) { e0 = e; fetch_entries(); }
        b = __builtin_amdgcn_readlane(blk, e - e0);
        const int x = __builtin_amdgcn_readlane(ex, e - e0);
        p.ek[i] = (int8_t)x;
        p.ev[i] = (int8_t)(x >> 8);
        p.tok[i] = __builtin_amdgcn_readlane(pg, e - e0) * a.P + sub * kTile;
      }
      if (b >= 0) {
        const unsigned char* at = a.pages + (((size_t)b * a.H + u.h) * tpp + sub) * kTileBytes + lane * 16;
        p.k[i][0] = load_stream16(at);
        p.k[i][1] = load_stream16(at + 1024);
        p.v[i][0] = load_stream16(at + kHalfTile);
        p.v[i][1] = load_stream16(at + kHalfTile + 1024);
      } else {
        p.tok[i] = kNowhere;
        p.ek[i] = p.ev[i] = kExpMin;
        p.k[i][0] = p.k[i][1] = p.v[i][0] = p.v[i][1] = make_uint4(0, 0, 0, 0);
      }
      ++t;
      if (++sub == tpp) { sub = 0; ++e; }
    }
  }

  // What products with keys of scale 2^e are taken times for logits in powers of two.  Never 0, which would make NaN of a hidden
  // product's -infinity (what that adds to a logit is below 2^-126 of its product), nor infinite, which would make it of a product
  // that is 0.
  __device__ __forceinline__ float logit_scale(int e) const {
    return __builtin_amdgcn_fmed3f(a.scale_log2 * two_to(e), 0x1p-126f, 0x1.fffffep127f);
  }
  // The products q k of the columns with a pair's tokens (four of each tile a lane): hides what a column does not see, and
  // raises the maxima where it has to.  ks: their logit_scale
  __device__ __forceinline__ void hide(f32x4 (&s)[NQ][2], const int (&tok)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tok[i] + kTile - 1 > u.pos0) {
#pragma unroll
        for (int g = 0; g < NQ; ++g)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (tok[i] + c * 4 + y > lim[g]) s[g][i][y] = -INFINITY;
      }
  }
  __device__ __forceinline__ void raise(const f32x4 (&s)[NQ][2], const float (&ks)[2]) {
    float mx[NQ];
    bool any = false;
#pragma unroll
    for (int g = 0; g < NQ; ++g) {             // (ks > 0 keeps the order)
      mx[g] = fmaxf(fmaxf(max3(s[g][0][0], s[g][0][1], s[g][0][2]), s[g][0][3]) * ks[0],
                    fmaxf(max3(s[g][1][0], s[g][1][1], s[g][1][2]), s[g][1][3]) * ks[1]);
      any |= mx[g] > m[g] - (kHead - kSlack);
    }
    if (__any(any)) {
#pragma unroll
      for (int g = 0; g < NQ; ++g) {
        mx[g] = fmaxf(mx[g], __shfl_xor(mx[g], 16, kWave));
        mx[g] = fmaxf(mx[g], __shfl_xor(mx[g], 32, kWave));
        // (a column that does not need it stays, so that no row's result depends on its neighbours)
        const float to = mx[g] > m[g] - (kHead - kSlack) ? mx[g] + kHead : m[g], down = __builtin_amdgcn_exp2f(m[g] - to);
        m[g] = to;
        l[g] *= down;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[g][i] *= down;
      }
    }
  }
  // The weights, as operands of the second product: rounded, and what that left
  __device__ __forceinline__ void soften(const f32x4 (&s)[NQ][2], const float (&ks)[2], uint4 (&w)[NQ][kParts]) {
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      float pr[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][i >> 2][i & 3], ks[i >> 2], -m[g]));
      l[g] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
      u32 x[4], rest[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = pack2<true>(pr[2 * i], pr[2 * i + 1]);
        if (DUP || TWO) rest[i] = pack2<true>(pr[2 * i] - as_f32(x[i] << 16), pr[2 * i + 1] - as_f32(x[i] & 0xffff0000u));
        if (DUP) x[i] = n & 8 ? rest[i] : x[i];
      }
      w[g][0] = make_uint4(x[0], x[1], x[2], x[3]);
      if constexpr (TWO) w[g][1] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
    }
  }

  __device__ __forceinline__ void take(const Pair& p) {
    f32x4 s[NQ][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int g = 0; g < NQ; ++g) s[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const auto k = widen<BF16>(word(p.k[i][j >> 1], (j & 1) * 2), word(p.k[i][j >> 1], (j & 1) * 2 + 1), 1.f, 1.f);
#pragma unroll
        for (int g = 0; g < NQ; ++g) s[g][i] = mfma32<BF16>(k, q[g][j], s[g][i]);
      }
    }
    const float ks[2] = {logit_scale(p.ek[0]), logit_scale(p.ek[1])};
    uint4 w[NQ][kParts];
    hide(s, p.tok);
    raise(s, ks);
    soften(s, ks, w);
    const float v0 = two_to(p.ev[0] - kValueDown), v1 = two_to(p.ev[1] - kValueDown);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x8 v = widen<true>(word(p.v[0][i >> 2], i & 3), word(p.v[1][i >> 2], i & 3), v0, v1);
#pragma unroll
      for (int x = 0; x < kParts; ++x)
#pragma unroll
        for (int g = 0; g < NQ; ++g) o[g][i] = mfma32<true>(v, __builtin_bit_cast(bf16x8, w[g][x]), o[g][i]);
    }
  }

  // The same for a stage of four tiles in LDS, already widened.  Operands are asked for four at a time, while the four before
  // them are taken.
  template <class Lds>
  __device__ __forceinline__ void take_staged(const Lds& lds, int stage) {
    typedef typename Op<BF16>::type op;
    uint4 b[2][4];
    // keys of tile 0 and 1, values of pair 0 in two halves, then the same of pair 1
    auto ask = [&](int i) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        b[i & 1][j] = i % 4 < 2 ? lds.k[stage][i / 4 * 2 + i % 4][j][lane] : lds.v[stage][i / 4][(i % 4 - 2) * 4 + j][lane];
      __builtin_amdgcn_sched_barrier(0);
    };
    ask(0);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      int tok[2], ek[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        tok[i] = __builtin_amdgcn_readfirstlane(lds.tok[stage][2 * x + i]);
        ek[i] = BF16 ? 0 : __builtin_amdgcn_readfirstlane(lds.ek[stage][2 * x + i]);
      }
      f32x4 s[NQ][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ask(4 * x + i + 1);
#pragma unroll
        for (int g = 0; g < NQ; ++g) s[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int g = 0; g < NQ; ++g) s[g][i] = mfma32<BF16>(__builtin_bit_cast(op, b[i][j]), q[g][j], s[g][i]);
      }
      float ks[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) ks[i] = logit_scale(BF16 ? kKeyDown : ek[i]);
      hide(s, tok);
      raise(s, ks);
      uint4 w[NQ][kParts];
      soften(s, ks, w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (4 * x + i + 3 < 8) ask(4 * x + i + 3);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int y = 0; y < kParts; ++y)
#pragma unroll
            for (int g = 0; g < NQ; ++g)
              o[g][i * 4 + j] = mfma32<true>(__builtin_bit_cast(bf16x8, b[i][j]), __builtin_bit_cast(bf16x8, w[g][y]), o[g][i * 4 + j]);
      }
    }
  }

  // Tiles [from, to) of the unit
  __device__ __forceinline__ void sweep(int from, int to) {
    if (from < to) {
      const int tpp = a.P / kTile;
      t = from; t1 = to;
      e = from / tpp;
      sub = from - e * tpp;
      e0 = e;
      fetch_entries();
      Pair p[2];
      load(p[0]);
      for (int left = to - from; left > 0; left -= 4) {
        load(p[1]);
        take(p[0]);
        if (left <= 2) break;
        load(p[0]);
        take(p[1]);
      }
    }
    close();
  }

  // Partial results of other workgroups, as this launch's lanes have them: accumulators [g][i][half][lane] in pairs, then
  // (maximum, sum) [g][n].  With DUP lanes n and n + 8 have the same.
  __device__ __forceinline__ u64* part_of(int slot) const { return a.part + (size_t)slot * part_words(NQ); }
  __device__ __forceinline__ void leave(int slot) const {
    u64* part = part_of(slot);
    if (DUP && (n & 8)) return;
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        store_agent(part + (g * 8 + i) * 2 * kWave + lane, pack_floats(o[g][i][0], o[g][i][1]));
        store_agent(part + ((g * 8 + i) * 2 + 1) * kWave + lane, pack_floats(o[g][i][2], o[g][i][3]));
      }
      if (c == 0) store_agent(part + NQ * 16 * kWave + g * 16 + n, pack_floats(m[g], l[g]));
    }
  }
  // The joined results slot(from), slot(from + step), ... of `count`
  template <class Slot>
  __device__ __forceinline__ void gather(int from, int step, int count, Slot slot) {
    const int mine = DUP ? lane & ~8 : lane;
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
        const u64 ml = load_agent(part + NQ * 16 * kWave + g * 16 + (mine & 15));
        u64 v[8][2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i][0] = load_agent(part + (g * 8 + i) * 2 * kWave + mine);
          v[i][1] = load_agent(part + ((g * 8 + i) * 2 + 1) * kWave + mine);
        }
        const float l2 = as_f32((u32)(ml >> 32)), m2 = l2 == 0.f ? kLowest : as_f32((u32)ml);
        const float to = fmaxf(m[g], m2), f1 = __builtin_amdgcn_exp2f(m[g] - to), f2 = l2 == 0.f ? 0.f : __builtin_amdgcn_exp2f(m2 - to);
        m[g] = to;
        l[g] = l[g] * f1 + l2 * f2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const f32x4 y = {as_f32((u32)v[i][0]), as_f32((u32)(v[i][0] >> 32)), as_f32((u32)v[i][1]), as_f32((u32)(v[i][1] >> 32))};
          o[g][i] = o[g][i] * f1 + y * f2;
        }
      }
    }
  }

  // Behind the last tile
  __device__ __forceinline__ void close() {
    // a column's four lanes have a quarter of its sum each
#pragma unroll
    for (int g = 0; g < NQ; ++g) {
      l[g] += __shfl_xor(l[g], 16, kWave);
      l[g] += __shfl_xor(l[g], 32, kWave);
      if (DUP)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) o[g][i][y] += __shfl_xor(o[g][i][y], 8, kWave);
    }
  }
};

// A column's result over all tokens
template <bool BF16, int N>
__device__ __forceinline__ void emit(const AttnArgs& a, const Unit& u, int r, int head, int d, const float (&v)[N], float m, float l) {
  const size_t at = (size_t)(u.row0 + r) * a.H * a.G + u.h * a.G + head;
  const float inv = l == 0.f ? 0.f : two_to(kValueDown) / l;
  u32 w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = pack2<BF16>(l == 0.f ? 0.f : v[2 * i] * inv, l == 0.f ? 0.f : v[2 * i + 1] * inv);
  if constexpr (N == 8) *reinterpret_cast<uint4*>(a.out + at * kHeadDim + d) = make_uint4(w[0], w[1], w[2], w[3]);
  else *reinterpret_cast<uint2*>(a.out + at * kHeadDim + d) = make_uint2(w[0], w[1]);
  if (a.lse != nullptr && d == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Where a piece's result goes: to the output if it is all of the unit (count == 1), else to slot `mine` of the partial
// results, which the last of the `count` pieces to arrive joins, in their order; slot(i) is the i-th one's number.
template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL>
__device__ __forceinline__ void emit_wave(const AttnArgs& a, const Wave<BF16, NQ, DUP, TWO, SEL>& w) {
#pragma unroll
  for (int g = 0; g < NQ; ++g) {
    int r, head;
    w.column(g, r, head);
    if (!w.real(r, head) || (DUP && (w.n & 8))) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v[4] = {w.o[g][i][0], w.o[g][i][1], w.o[g][i][2], w.o[g][i][3]};
      emit<BF16>(a, w.u, r, head, i * 16 + w.c * 4, v, w.m[g], w.l[g]);
    }
  }
}
template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL, class Slot>
__device__ __forceinline__ void finish_wave(const AttnArgs& a, Wave<BF16, NQ, DUP, TWO, SEL>& w, int count, int mine, int ticket, Slot slot) {
  if (count > 1) {
    w.leave(mine);                             // (written through and drained before the ticket, and read past the caches: no fence
    wave_drain_memory();                       // of the ticket's, which would empty an XCD's L2: 583 us for 533 with it)
    int before = 0;
    if (w.lane == 0) before = __hip_atomic_fetch_add(a.ticket + ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    before = __builtin_amdgcn_readfirstlane(before);
    if (before != count - 1) return;
    if (w.lane == 0) store_agent(a.ticket + ticket, 0);
    w.gather(0, 1, count, slot);
  }
  emit_wave(a, w);
}

template <int NQ>
struct AttnLds {
  float ml[kAttnWaves][16 * NQ][2];
  __align__(16) float o[kAttnWaves][16][kColFloats];
  int last;
};

// The waves' results of one unit as one: with to_slot < 0 to the output, else there
template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL>
__device__ __forceinline__ void merge_waves(const AttnArgs& a, const Wave<BF16, NQ, DUP, TWO, SEL>& w, AttnLds<NQ>& lds, int to_slot) {
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
    for (int i = 0; i < 8; ++i) *reinterpret_cast<f32x4*>(&lds.o[wave][w.n][i * 16 + w.c * 4]) = w.o[g][i] * f;
    __syncthreads();
    const int n = tid >> 4, d = (tid & 15) * 8;   // a column and eight of its elements
    const int col = g * 16 + n;
    int r = 0, head = n;
    if (!DUP) { r = col / a.G; head = col - r * a.G; }
    if (w.real(r, head) && !(DUP && n >= 8)) {
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
        const int at = (g * 8 + d / 16) * 2 * kWave + d % 16 / 4 * 16 + n;   // as lanes d % 16 / 4 * 16 + n and 16 more leave it
#pragma unroll
        for (int y = 0; y < 4; ++y) store_agent(part + at + (y & 1) * kWave + (y >> 1) * 16, pack_floats(v[2 * y], v[2 * y + 1]));
        if (d == 0) store_agent(part + NQ * 16 * kWave + col, pack_floats(top, L));
      }
    }
  }
}
// The same as finish_wave for a piece that the waves of the workgroup shared
template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL, class Slot>
__device__ __forceinline__ void finish_group(const AttnArgs& a, Wave<BF16, NQ, DUP, TWO, SEL>& w, AttnLds<NQ>& lds, int count, int mine,
                                             int ticket, Slot slot) {
  merge_waves(a, w, lds, count == 1 ? -1 : mine);
  if (count == 1) return;
  wave_drain_memory();
  __syncthreads();
  if (threadIdx.x == 0) {
    lds.last = __hip_atomic_fetch_add(a.ticket + ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1;
    if (lds.last) store_agent(a.ticket + ticket, 0);
  }
  __syncthreads();
  if (!lds.last) return;
  w.gather(threadIdx.x / kWave, kAttnWaves, count, slot);
  merge_waves(a, w, lds, -1);
}

// Tiles [t0, t1) of a unit: by all waves, or, a short unit, by wave `solo` alone.
template <bool BF16, int NQ, bool DUP, bool TWO, bool SEL, class Slot>
__device__ __forceinline__ void piece(const AttnArgs& a, Wave<BF16, NQ, DUP, TWO, SEL>& w, AttnLds<NQ>& lds, const Unit& u, int t0, int t1,
                                      int solo, int count, int mine, int ticket, Slot slot) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (!SEL) t1 = min(t1, max(t0, (u.pos0 + u.rows - 1) / kTile + 1));   // none of the rows sees more
  if (count == 1 && t1 - t0 < kCoopTiles) {    // (pieces of one unit are joined in one way, whichever comes last: the sums' order is fixed)
    if (wave != solo) return;
    w.begin(u);
    w.sweep(t0, t1);
    emit_wave(a, w);
  } else {
    const int per = ((t1 - t0 + 1) / 2 + kAttnWaves - 1) / kAttnWaves * 2;
    w.begin(u);
    w.sweep(min(t0 + wave * per, t1), min(t0 + (wave + 1) * per, t1));
    finish_group(a, w, lds, count, mine, ticket, slot);
  }
}

// All tokens.  The units' tiles, one unit behind the other, are dealt out evenly: workgroup i has tiles [i, i + 1) * chunk of
// them all, wherever units begin and end in there, so that lengths of any kind keep all CUs busy to the end.  A unit is up to
// a.R rows of a sequence and a head; `each(u, t0, t1, f, count, mine, slot)` takes tiles [t0, t1) of one:
// one of `count` pieces, whose partial result goes to slot `mine`; f numbers the unit's ticket.
__device__ __forceinline__ u64 uniform(u64 x) {
  return (u64)(u32)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (u32)__builtin_amdgcn_readfirstlane((int)x);
}
// The first unit of a sequence has `first` tiles and every next one `more` more, which is what their last rows see, rounded up.
template <int NT, class Each>
__device__ __forceinline__ void deal(const AttnArgs& a, bool grow, Each each) {
  __shared__ u64 scan[NT / kWave];
  __shared__ u64 s_base;
  __shared__ int s_seq;
  const int tid = threadIdx.x, lane = tid % kWave, wv = tid / kWave;
  const int more = grow ? (a.R + kTile - 1) / kTile : 0;
  auto of = [&](int b, int& row0, int& rows, int& len, int& first) {   // returns units a head
    row0 = min(max(a.row_start[b], 0), a.T);
    rows = min(max(a.row_start[b + 1], row0), a.T) - row0;
    len = min(max(a.kv_len[b], 0), a.NP * a.P);
    first = max(((grow ? min(len, max(len - rows, 0) + a.R) : len) + kTile - 1) / kTile, 1);
    return (rows + a.R - 1) / a.R;
  };
  // tiles of a sequence's first n units of a head
  auto upto_unit = [&](u64 n, int first) { return n * first + n * (n - 1) / 2 * more; };
  const int per = (a.B + NT - 1) / NT, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  u64 mine = 0;
  for (int b = b0; b < b1; ++b) {
    int row0, rows, len, first;
    const u64 units = of(b, row0, rows, len, first);
    mine += upto_unit(units, first) * a.H;
  }
  u64 upto = mine;
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    const u64 y = ((u64)__shfl_up((u32)(upto >> 32), x, kWave) << 32) | __shfl_up((u32)upto, x, kWave);
    if (lane >= x) upto += y;
  }
  if (lane == kWave - 1) scan[wv] = upto;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int i = 0; i < NT / kWave; ++i) {
    if (i < wv) upto += scan[i];
    all += scan[i];
  }
  u64 chunk = (all + a.W - 1) / a.W;
  if (chunk < (u64)kLeastTiles) chunk = kLeastTiles;
  // neighbours in the order of the units share keys and values: they go to one XCD, whose workgroups are every eighth, and its L2
  const int groups = (int)((all + chunk - 1) / chunk), each_xcd = (groups + kXcds - 1) / kXcds;
  if ((int)blockIdx.x / kXcds >= each_xcd) return;
  const int group = blockIdx.x % kXcds * each_xcd + blockIdx.x / kXcds;
  const u64 lo = group * chunk, hi = min(lo + chunk, all);
  if (lo >= all) return;
  if (upto - mine <= lo && lo < upto) {
    u64 base = upto - mine;
    int b = b0;
    for (; b < b1; ++b) {
      int row0, rows, len, first;
      const u64 units = of(b, row0, rows, len, first);
      const u64 n = upto_unit(units, first) * a.H;
      if (lo < base + n) break;
      base += n;
    }
    s_base = base;
    s_seq = b;
  }
  __syncthreads();
  u64 at = uniform(lo), base = uniform(s_base);
  const u64 per_group = uniform(chunk), stop = uniform(hi);
  int b = __builtin_amdgcn_readfirstlane(s_seq);
  while (at < stop && b < a.B) {
    int row0, rows, len, first;
    const int units = __builtin_amdgcn_readfirstlane(of(b, row0, rows, len, first));
    row0 = __builtin_amdgcn_readfirstlane(row0);
    rows = __builtin_amdgcn_readfirstlane(rows);
    len = __builtin_amdgcn_readfirstlane(len);
    first = __builtin_amdgcn_readfirstlane(first);
    const u64 end = base + upto_unit(units, first) * a.H;
    while (at < min(end, stop)) {
      // unit `part` of its head: the largest one that begins at or before `at`, a head's units one behind the other
      const u64 of_head = upto_unit(units, first), x = at - base, h = x / of_head, in = x - h * of_head;
      u64 part;
      if (more == 0) part = in / first;
      else {                                   // first n + more n (n - 1) / 2 <= in, put right by whole numbers
        const float p = first - 0.5f * more;
        part = (u64)fmaxf((sqrtf(p * p + 2.f * more * (float)in) - p) / more, 0.f);
        while (part > 0 && upto_unit(part, first) > in) --part;
        while (upto_unit(part + 1, first) <= in) ++part;
        part = uniform(part);
      }
      const u64 begin = base + h * of_head + upto_unit(part, first);
      const int tiles = first + (int)part * more, t0 = (int)(at - begin), t1 = (int)min((u64)tiles, stop - begin);
      Unit u;
      u.seq = b;
      u.h = (int)h;
      u.row0 = row0 + (int)part * a.R;
      u.rows = min(a.R, rows - (int)part * a.R);
      u.pos0 = len - rows + (int)part * a.R;
      u.entries = min((len + a.P - 1) / a.P, a.NP);
      const int f = (int)(begin / per_group), count = (int)((begin + tiles - 1) / per_group) - f + 1;
      // a workgroup has the beginning of one unit that goes on behind it, and at most one piece that began before it
      each(u, t0, t1, f, count, group * 2 + (t0 == 0 ? 1 : 0), [f](int x) { return x == 0 ? f * 2 + 1 : (f + x) * 2; });
      at = begin + t1;
    }
    base = end;
    ++b;
  }
}

// A few rows of a sequence (up to 16 NQ columns): each wave has all of them and a part of the tokens, with a pair of tiles on its
// way behind the one it takes.  Bound by the memory: 16 x 32768 tokens of 8 heads 167 us (6.4 TB/s), 24 ragged contexts with up to
// three rows of 7 x 4 heads 104 us (5.1 TB/s); short contexts by their chain of trips to memory (4 x 1000 tokens 14.5 us).
template <bool BF16, int NQ, bool DUP>
__global__ __launch_bounds__(kAttnThreads, 2) void q8_attn_dense_kernel(AttnArgs a) {
  __shared__ AttnLds<NQ> lds;
  Wave<BF16, NQ, DUP, !DUP, false> w(a);
  int solo = 0;
  deal<kAttnThreads>(a, false, [&](const Unit& u, int t0, int t1, int f, int count, int mine, auto slot) {
    piece(a, w, lds, u, t0, t1, solo, count, mine, f, slot);
    solo = (solo + 1) % kAttnWaves;
  });
}

// Many rows of a sequence: each wave has its own kRowGroups * 16 columns, and the workgroup goes through the tokens together,
// 64 at a time: every wave fetches one tile, widens it and puts it into LDS in operand order, while the 64 before it are
// taken; so a code is widened once for four waves.  Bound by the matrix cores and the vector unit alike, which two waves a SIMD hardly
// get to work at the same time: 2 x 2048 rows of 32/8 heads behind 6144 tokens 530 us (910 TFLOP/s).  With 48 columns a wave
// registers spill (818 us), with 64 and a SIMD's registers for one wave the vector unit's values land in accumulation registers
// (800), with 32 a widened code serves fewer columns, but all fits.
constexpr int kRowGroups = 2;
constexpr int kStageTiles = kAttnWaves;
struct RowsLds {
  uint4 k[2][kStageTiles][4][kWave];           // [stage][tile][32 elements][lane], in the type of q
  uint4 v[2][kStageTiles / 2][8][kWave];       // [stage][pair of tiles][16 elements][lane], in bf16
  int tok[2][kStageTiles], ek[2][kStageTiles];
};

template <bool BF16>
__global__ __launch_bounds__(kAttnThreads, 2) void q8_attn_rows_kernel(AttnArgs a) {
  constexpr int NQ = kRowGroups;
  __shared__ RowsLds lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Wave<BF16, NQ, false, !BF16, false> w(a);
  const int tpp = a.P / kTile, rows = a.R / kAttnWaves;                // tiles of a page; rows of a wave
  deal<kAttnThreads>(a, true, [&](const Unit& whole, int t0, int t1, int f, int count, int mine, auto slot) {
    Unit u = whole;                            // this wave's rows
    u.row0 += wave * rows;
    u.pos0 += wave * rows;
    u.rows = min(max(whole.rows - wave * rows, 0), rows);
    const int last = u.pos0 + u.rows - 1;      // position of its last row
    w.begin(u);
    t1 = min(t1, max(t0, (whole.pos0 + whole.rows - 1) / kTile + 1));  // none of the rows sees more
    uint4 raw[4];
    int tok = kNowhere, ek = kExpMin, ev = kExpMin, e0 = -kWave, blk = -1, ex = 0;
    auto fetch = [&](int t) {                  // this wave's tile of the stage that begins with tile t
      t += wave;
      int b = -1;
      ek = ev = kExpMin;
      if (t < t1) {
        const int e = t / tpp, sub = t - e * tpp;
        if (e - e0 >= kWave) {                 // blocks and exponents of the next 64 pages
          e0 = e;
          const int i = e0 + w.lane;
          blk = i < whole.entries ? a.table[(size_t)whole.seq * a.NP + i] : -1;
          if ((unsigned)blk >= (unsigned)a.NB) blk = -1;
          ex = blk >= 0 ? *reinterpret_cast<const int16_t*>(a.exps + ((size_t)blk * a.H + whole.h) * 2) : 0;
        }
        b = __builtin_amdgcn_readlane(blk, e - e0);
        if (b >= 0) {
          const int x = __builtin_amdgcn_readlane(ex, e - e0);
          ek = (int8_t)x;
          ev = (int8_t)(x >> 8);
          const unsigned char* at = a.pages + (((size_t)b * a.H + whole.h) * tpp + sub) * kTileBytes + w.lane * 16;
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const uint4*>(at + i * 1024);
        }
      }
      tok = b >= 0 ? t * kTile : kNowhere;
    };
    auto put = [&](int s) {                    // zeros where there is no tile: no column sees it, but it has to be finite
      if (tok == kNowhere)
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = make_uint4(0, 0, 0, 0);
      // (bf16 has the range to take the keys' scale in; f16 has not, and it goes into the logits)
      const float sk = BF16 ? two_to(ek - kKeyDown) : 1.f, sv = two_to(ev - kValueDown);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        lds.k[s][wave][j][w.lane] = __builtin_bit_cast(uint4, widen<BF16>(word(raw[j >> 1], (j & 1) * 2), word(raw[j >> 1], (j & 1) * 2 + 1), sk, sk));
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint4 x = __builtin_bit_cast(uint4, widen<true>(word(raw[2 + (i >> 2)], i & 3), word(raw[2 + (i >> 2)], (i & 3) + 1), sv, sv));
        u64* to = reinterpret_cast<u64*>(&lds.v[s][wave >> 1][i][w.lane]) + (wave & 1);
        to[0] = (u64)x.y << 32 | x.x;
        to[2 * kWave] = (u64)x.w << 32 | x.z;  // (the next 16 elements' operand)
      }
      if (w.lane == 0) { lds.tok[s][wave] = tok; lds.ek[s][wave] = ek; }
    };
    __syncthreads();                           // (the last piece's stages have been read)
    if (t0 < t1) {
      fetch(t0);
      put(0);
      __syncthreads();
      int s = 0;
      for (int t = t0; t < t1; t += kStageTiles, s ^= 1) {
        const bool more = t + kStageTiles < t1;
        if (more) fetch(t + kStageTiles);
        if (u.rows > 0 && t * kTile <= last) w.take_staged(lds, s);
        if (more) {
          put(s ^ 1);
          __syncthreads();
        }
      }
    }
    w.close();
    finish_wave(a, w, count, mine * kAttnWaves + wave, f * kAttnWaves + wave, [&](int x) { return slot(x) * kAttnWaves + wave; });
  });
}

// Selected pages: a unit is one row and head, in S pieces, so that there are two workgroups for each CU.  16 x 8 units of 256 pages
// 29 us (4.6 TB/s): the memory behind a chain of selection, table, exponents and pages.
template <bool BF16>
__global__ __launch_bounds__(kAttnThreads, 2) void q8_attn_selected_kernel(AttnArgs a) {
  __shared__ AttnLds<1> lds;
  Unit u;
  u.row0 = blockIdx.x;
  u.h = blockIdx.y / a.S;
  const int s = blockIdx.y - u.h * a.S, unit = u.row0 * a.H + u.h;
  u.rows = 1;
  u.seq = a.row_seq[u.row0];
  u.pos0 = a.row_pos[u.row0];
  if ((unsigned)u.seq >= (unsigned)a.B || u.pos0 < 0 || u.pos0 >= a.NP * a.P) return;
  u.entries = min(a.k, u.pos0 / a.P + 1);
  const int tiles = u.entries * (a.P / kTile), per = (tiles + a.S - 1) / a.S;
  Wave<BF16, 1, true, false, true> w(a);
  piece(a, w, lds, u, min(s * per, tiles), min((s + 1) * per, tiles), 0, a.S, unit * a.S + s, unit,
        [&](int x) { return unit * a.S + x; });
}

// Columns of 16 that the rows of a sequence take, on the average: 1 and 2 go to waves that share the tokens, 0 (more) to
// waves that share the columns
static int column_groups(int T, int B, int G) {
  const int64_t want = (int64_t)((T + B - 1) / B) * G;
  return want <= 16 ? 1 : want <= 32 ? 2 : 0;
}
// 8-byte words of a workgroup's partial results: two pieces, of each wave where the waves have columns of their own
static int64_t part_words_of_group(int T, int B, int G) {
  const int groups = T <= B ? 1 : column_groups(T, B, G);
  return 2 * (int64_t)(groups ? part_words(groups) : kAttnWaves * part_words(kRowGroups));
}

}  // namespace q8
}  // namespace kvd

int64_t kvd_q8_attn_bytes(const kvd_q8_cache* c, const kvd_q8_rows* r) {
  using namespace kvd::q8;
  static_assert(kAttnGroups * kAttnWaves * 4 <= kTicketBytes, "a ticket for each wave of each workgroup");
  return kTicketBytes + (int64_t)kAttnGroups * 8 * part_words_of_group(r->n_rows, r->n_seqs, c->n_q_heads / c->n_kv_heads);
}

extern "C" int kvd_q8_attn(const kvd_q8_cache* c, const kvd_q8_rows* r, const void* q, int64_t q_stride, const int32_t* sel_pages,
                           int32_t topk_pages, void* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace kvd::q8;
  using kvd::kHeadDim;
  if (int e = check_cache(c, r)) return e;
  if (!stride_ok(q_stride, c->n_q_heads)) return KVD_ERR_SHAPE;
  if (sel_pages != nullptr && (topk_pages < 1 || topk_pages > KVD_MAX_TOPK)) return KVD_ERR_SHAPE;
  if (!aligned(c->pages, 16) || !aligned(c->exps, 2) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16)) return KVD_ERR_ARG;
  if (out == q) return KVD_ERR_ARG;            // (a row's pieces read q while the first unit that is done writes)
  if ((reinterpret_cast<uintptr_t>(lse) & 3) || (reinterpret_cast<uintptr_t>(sel_pages) & 3)) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->kv_len, 4) || !aligned(r->row_start, 4) || !aligned(r->row_seq, 4) || !aligned(r->row_pos, 4)) return KVD_ERR_ARG;
  if (workspace_bytes < kvd_q8_attn_bytes(c, r)) return KVD_ERR_CAPACITY;
  kvd::q8::AttnArgs a;
  a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
  a.table = r->page_table; a.kv_len = r->kv_len; a.row_start = r->row_start; a.row_seq = r->row_seq; a.row_pos = r->row_pos;
  a.sel = sel_pages;
  a.pages = static_cast<const unsigned char*>(c->pages); a.exps = c->exps;
  a.out = static_cast<uint16_t*>(out); a.lse = lse;
  a.ticket = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<kvd::u64*>(static_cast<char*>(workspace) + kTicketBytes);
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.H = c->n_kv_heads; a.G = c->n_q_heads / c->n_kv_heads;
  a.P = c->page_size; a.NB = c->n_blocks; a.k = topk_pages;
  a.W = kAttnGroups;
  a.scale_log2 = (c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)kHeadDim)) * kLog2e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = c->kv_dtype == KVD_BF16;
  if (sel_pages != nullptr) {
    const int64_t units = (int64_t)a.T * a.H;
    const int tiles = topk_pages * (a.P / kTile);
    int S = (int)(kAttnGroups / units);
    if (S > tiles / kLeastTiles) S = tiles / kLeastTiles;
    a.S = S < 1 ? 1 : S;
    a.R = 1;
    const dim3 grid(a.T, a.H * a.S);
    if (bf16) hipLaunchKernelGGL(q8_attn_selected_kernel<true>, grid, dim3(kAttnThreads), 0, s, a);
    else hipLaunchKernelGGL(q8_attn_selected_kernel<false>, grid, dim3(kAttnThreads), 0, s, a);
    return launched();
  }
  a.S = 1;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.W), dim3(kAttnThreads), 0, s, a); };
  if (a.T <= a.B) {
    a.R = 1;
    if (bf16) go(q8_attn_dense_kernel<true, 1, true>); else go(q8_attn_dense_kernel<false, 1, true>);
    return launched();
  }
  const int groups = column_groups(a.T, a.B, a.G);
  a.R = groups ? 16 * groups / a.G : 16 * kRowGroups / a.G * kAttnWaves;
  if (bf16) {
    if (groups == 1) go(q8_attn_dense_kernel<true, 1, false>);
    else if (groups == 2) go(q8_attn_dense_kernel<true, 2, false>);
    else go(q8_attn_rows_kernel<true>);
  } else {
    if (groups == 1) go(q8_attn_dense_kernel<false, 1, false>);
    else if (groups == 2) go(q8_attn_dense_kernel<false, 2, false>);
    else go(q8_attn_rows_kernel<false>);
  }
  return launched();
}
