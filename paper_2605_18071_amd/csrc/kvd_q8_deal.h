// How the attention kernels of the paged caches deal out the tokens of all sequences to their workgroups.
#pragma once
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kXcds = 8;
constexpr int kAllTiles = 1 << 30;             // no bound on a unit's tiles

// What the rows of one unit (up to R rows of a sequence, one head) have in common
struct Unit {
  int row0, rows, h, seq, pos0, entries;       // pos0: position of row0; entries: pages (or selected pages)
  int lead;                                    // tiles in front of those that were counted
};

// All tokens.  The units' tiles, one unit behind the other, are dealt out evenly: workgroup i has tiles [i, i + 1) * chunk of
// them all, wherever units begin and end in there, so that lengths of any kind keep all CUs busy to the end.  A unit is up to
// a.R rows of a sequence and a head; `each(u, t0, t1, f, count, mine, slot)` takes tiles [t0, t1) of one:
// one of `count` pieces, whose partial result goes to slot `mine`; f numbers the unit's ticket.
__device__ __forceinline__ u64 uniform(u64 x) {
  return (u64)(u32)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (u32)__builtin_amdgcn_readfirstlane((int)x);
}
// The first unit of a sequence has `first` tiles and every next one `more` more, which is what their last rows see, rounded up.
// `most` bounds the tiles of a unit; a.W workgroups (a multiple of kXcds) have LEAST tiles at least.  ALIGN > 0: if the units are few
// enough for a workgroup to each ALIGN tiles of one, that is how they are dealt out (not where they grow): then a unit of no more than
// that needs no joining, which takes longer than its tiles.  lead(row): tiles at the beginning of the sequence that begins with that
// row which are left out of the count.  PAD (less than LEAST): what a unit costs
// whatever its length, in tiles, which it counts for at its beginning; a share that would begin in there begins with the unit.
template <int NT, int LEAST, int ALIGN, int PAD, class Args, class Lead, class Each>
__device__ __forceinline__ void deal(const Args& a, bool grow, int most, Lead lead, Each each) {
  __shared__ u64 scan[NT / kWave];
  __shared__ u64 s_base;
  __shared__ int s_seq;
  const int tid = threadIdx.x, lane = tid % kWave, wv = tid / kWave;
  const int more = grow ? (a.R + kTile - 1) / kTile : 0;
  int align = 1, pad = PAD;                    // what a unit's tiles are rounded up to, and what they are preceded by
  int skip = 0;                                // lead of the sequence that was last asked for
  auto of = [&](int b, int& row0, int& rows, int& len, int& first) {   // returns units a head
    row0 = min(max(a.row_start[b], 0), a.T);
    rows = min(max(a.row_start[b + 1], row0), a.T) - row0;
    len = min(max(a.kv_len[b], 0), a.NP * a.P);
    first = max(((grow ? min(len, max(len - rows, 0) + a.R) : len) + kTile - 1) / kTile, 1);
    skip = rows > 0 ? min(lead(row0), first - 1) : 0;
    first = min(first - skip, most) + pad;
    if (ALIGN > 0) first = (first + align - 1) / align * align;
    return (rows + a.R - 1) / a.R;
  };
  // tiles of a sequence's first n units of a head
  auto upto_unit = [&](u64 n, int first) { return n * first + n * (n - 1) / 2 * more; };
  const int per = (a.B + NT - 1) / NT, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  u64 mine, upto, all;                         // tiles of this thread's sequences, up to their last, of all
  auto count = [&] {
    mine = all = 0;
    for (int b = b0; b < b1; ++b) {
      int row0, rows, len, first;
      const u64 units = of(b, row0, rows, len, first);
      mine += upto_unit(units, first) * a.H;
    }
    upto = mine;
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) {
      const u64 y = ((u64)__shfl_up((u32)(upto >> 32), x, kWave) << 32) | __shfl_up((u32)upto, x, kWave);
      if (lane >= x) upto += y;
    }
    if (lane == kWave - 1) scan[wv] = upto;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / kWave; ++i) {
      if (i < wv) upto += scan[i];
      all += scan[i];
    }
  };
  if (ALIGN > 0 && !grow) {
    align = ALIGN;
    pad = 0;
    count();
    if (all > (u64)a.W * ALIGN) {
      align = 1;
      pad = PAD;
      __syncthreads();                         // (the sums have been read)
      count();
    }
  } else count();
  u64 chunk = (all + a.W - 1) / a.W;
  if (chunk < (u64)LEAST) chunk = LEAST;
  if (ALIGN > 0 && align > 1) chunk = ALIGN;
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
    const int in_front = __builtin_amdgcn_readfirstlane(skip);
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
      const int tiles = first + (int)part * more;
      int t0 = (int)(at - begin), t1 = (int)min((u64)tiles, stop - begin), f = (int)(begin / per_group);
      const int last = (int)((begin + tiles - 1) / per_group);
      at = begin + t1;
      if (PAD > 0 && pad > 0) {
        static_assert(PAD < LEAST, "");
        if (t1 <= pad && t1 < tiles) break;    // (the next workgroup begins with the unit)
        f = (int)((begin + pad) / per_group);
        t0 = max(t0 - pad, 0);
        t1 -= pad;
      }
      const int count = last - f + 1;
      Unit u;
      u.lead = in_front;
      u.seq = b;
      u.h = (int)h;
      u.row0 = row0 + (int)part * a.R;
      u.rows = min(a.R, rows - (int)part * a.R);
      u.pos0 = len - rows + (int)part * a.R;
      u.entries = min((len + a.P - 1) / a.P, a.NP);
      // a workgroup has the beginning of one unit that goes on behind it, and at most one piece that began before it
      each(u, t0, t1, f, count, group * 2 + (t0 == 0 ? 1 : 0), [f](int x) { return x == 0 ? f * 2 + 1 : (f + x) * 2; });
    }
    base = end;
    ++b;
  }
}

}  // namespace q8
}  // namespace kvd
