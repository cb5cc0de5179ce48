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
// stays, and stored whole, 16 bytes a lane.  Bound by the memory: 32768 tokens of 8 heads 35 us, which is what a copy of as many bytes
// takes.  (A wave a tile without barriers: 37, and 10 for 8 where a step has 10000 tokens.)
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

constexpr int kReadThreads = 256, kReadRows = 16;      // a wave has 16 rows
constexpr u32 kNoLine = 0xffffffffu;
constexpr int kReadHeads = 2;                  // heads of a wave (20 k tokens of 8 heads with the call: 23.7 us; with one 27.4, with four 26.2)

struct ReadArgs {
  uint16_t *k, *v;
  long long k_stride, v_stride;
  const int32_t *table, *row_seq, *row_pos;
  const unsigned char* pages;
  int B, NP, T, H, P, NB;
};

// Codes i and i + 1 (i even) of eight to two elements; f16 has no 6 * 2^14: the largest number it has stands for more
template <bool BF16, int BYTE>
__device__ __forceinline__ u32 widen2(u32 codes, float scale) {
  if constexpr (BF16) return __builtin_bit_cast(u32, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
  else {
    const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, BYTE);
    return pack2<false>(fminf(fmaxf(x[0], -65504.f), 65504.f), fminf(fmaxf(x[1], -65504.f), 65504.f));
  }
}

// Keys lie in the order of their elements: 16 lanes have a token, four tokens at a time.  Values lie by element, all tokens of a tile in
// 8 bytes: neighbouring lanes exchange theirs, so that each has two elements that follow each other, and 64 lanes write a
// token whole.  Rows that follow each other in a tile take it together; any others have a turn of their own, and a trip to memory in it: 64 rows of
// one sequence 5.7 us, of as many sequences 11.1; 16384 rows in pieces 15, by chance 39.
// HP heads have their rows looked up once, and are on their way together.  Bound by the memory: 20 k tokens of 8 heads to f16 18.6 us (5.6
// TB/s), 300 tokens 6.0 (rows, table, tile: three trips one behind the other).
template <bool BF16, int HP>
__global__ __launch_bounds__(kReadThreads) void read_kernel(ReadArgs a) {
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned of_heads = (a.H + HP - 1) / HP, unit = blockIdx.x * (kReadThreads / kWave) + wave, group = unit / of_heads;
  const int h0 = (unit - group * of_heads) * HP, tpp = a.P / kTile;
  const long long row0 = (long long)group * kReadRows;
  if (row0 >= a.T) return;
  // lane i: row i's tile of head 0, in lines, and its token in there
  u32 line = kNoLine;
  int pos = -1;
  if (lane < kReadRows && row0 + lane < a.T) {
    const int seq = a.row_seq[row0 + lane];
    pos = a.row_pos[row0 + lane];
    if ((unsigned)seq < (unsigned)a.B && pos >= 0 && pos < a.NP * a.P) {
      const int block = a.table[(size_t)seq * a.NP + pos / a.P];
      if ((unsigned)block < (unsigned)a.NB) line = ((u32)block * a.H * tpp + pos % a.P / kTile) * (kTileBytes / 128);
    }
  }
  const u32 before = __shfl_up(line, 1, kWave);
  const int pos_before = __shfl_up(pos, 1, kWave);
  // bit i: whether there is a row i, and whether it follows the one before it in a tile
  const u32 there = (u32)__ballot(line != kNoLine) & 0xffffu;
  const u32 follows = (u32)__ballot(lane > 0 && line == before && pos == pos_before + 1 && pos % kTile != 0) & 0xffffu;
  auto tile_of = [&](u32 first, int i) {       // of the i-th head; of the last one where there are no more
    return a.pages + ((size_t)first + (size_t)min(h0 + i, a.H - 1) * tpp * (kTileBytes / 128)) * 128;
  };
  {
    const int t0 = lane >> 4, j = lane & 15;
    u32 codes[HP][4];
    unsigned char scale[HP][4];
    bool ok[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * i + t0, at = __shfl(pos, r, kWave);
      const u32 first = __shfl(line, r, kWave);
      ok[i] = first != kNoLine;
      const int t = ok[i] ? at % kTile : 0;
#pragma unroll
      for (int y = 0; y < HP; ++y) {
        const unsigned char* tile = tile_of(ok[i] ? first : 0u, y);
        codes[y][i] = *reinterpret_cast<const u32*>(tile + t * 64 + j * 4);
        scale[y][i] = tile[kKeyScales + (j >> 2) * 16 + (t & 3) * 4 + (t >> 2)];
      }
    }
#pragma unroll
    for (int y = 0; y < HP; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (ok[i] && h0 + y < a.H) {
          const float s = two_to((int)scale[y][i] - kBias);
          *reinterpret_cast<uint4*>(a.k + (row0 + 4 * i + t0) * a.k_stride + (h0 + y) * kHeadDim + j * 8) =
              make_uint4(widen2<BF16, 0>(codes[y][i], s), widen2<BF16, 1>(codes[y][i], s), widen2<BF16, 2>(codes[y][i], s), widen2<BF16, 3>(codes[y][i], s));
        }
  }
  const int x = lane >> 4, n = lane & 15, odd = lane & 1;
  const int d = 32 * x + (odd ? 16 + n - 1 : n);         // the first of the lane's two elements
  for (u32 left = there & ~follows; left; left &= left - 1) {
    const int r0 = __builtin_ctz(left);
    const u32 stops = ~(follows & there) >> r0 >> 1;
    const int count = __builtin_ctz(stops | 0x10000u >> r0 >> 1) + 1;
    const int t0 = __builtin_amdgcn_readlane(pos, r0) % kTile;
    uint4 mine[HP], scales[HP];
#pragma unroll
    for (int y = 0; y < HP; ++y) {
      const unsigned char* tile = tile_of((u32)__builtin_amdgcn_readlane((int)line, r0), y);
      mine[y] = *reinterpret_cast<const uint4*>(tile + kValues + lane * 16);
      scales[y] = *reinterpret_cast<const uint4*>(tile + kValueScales + x * 16);
    }
#pragma unroll
    for (int y = 0; y < HP; ++y) {
      if (h0 + y >= a.H) break;
      // elements n and n + 16 of 32: even lanes take the first of theirs and their neighbour's, odd ones the second
      const u32 give0 = odd ? mine[y].x : mine[y].z, give1 = odd ? mine[y].y : mine[y].w;
      const u32 got0 = (u32)__builtin_amdgcn_update_dpp(0, (int)give0, 0xB1, 0xf, 0xf, true);
      const u32 got1 = (u32)__builtin_amdgcn_update_dpp(0, (int)give1, 0xB1, 0xf, 0xf, true);
      const u32 lo[2] = {odd ? got0 : mine[y].x, odd ? got1 : mine[y].y}, hi[2] = {odd ? mine[y].z : got0, odd ? mine[y].w : got1};
      const u32 sc[4] = {scales[y].x, scales[y].y, scales[y].z, scales[y].w};
      uint16_t* to = a.v + (row0 + r0 - t0) * a.v_stride + (h0 + y) * kHeadDim + d;
#pragma unroll
      for (int t = 0; t < kTile; ++t)
        if (t >= t0 && t < t0 + count) {
          const u32 c = (lo[t >> 3] >> (4 * (t & 7)) & 15) | (hi[t >> 3] >> (4 * (t & 7)) & 15) << 4;
          *reinterpret_cast<u32*>(to + t * a.v_stride) = widen2<BF16, 0>(c, two_to((int)(sc[t >> 2] >> (8 * (t & 3)) & 255) - kBias));
        }
    }
  }
}

template <bool BF16>
static void launch_read(const ReadArgs& a, hipStream_t s) {
  const unsigned groups = (a.T + kReadRows - 1) / kReadRows, waves = kReadThreads / kWave;
  auto go = [&](auto kernel, unsigned of_heads) { hipLaunchKernelGGL(kernel, dim3((groups * of_heads + waves - 1) / waves), dim3(kReadThreads), 0, s, a); };
  // few waves have a head each, to be many: 4000 tokens of 8 heads 9.3 us, 10.6 with two
  if (a.H >= kReadHeads && (uint64_t)groups * a.H >= 4096) go(read_kernel<BF16, kReadHeads>, (a.H + kReadHeads - 1) / kReadHeads);
  else go(read_kernel<BF16, 1>, a.H);
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c->kv_dtype == KVD_BF16) launch_read<true>(a, s);
  else launch_read<false>(a, s);
  return launched();
}
