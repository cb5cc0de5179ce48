// Page tables and slot maps of a step, built on the GPU from the requests' lengths: three prefix sums over the
// sequences (rows, runs, pages begun), then every row, run and new page finds its sequence in them by bisection.
// Everything is a few bytes an item: the time is the launch and a handful of dependent trips to memory and LDS (6.4 us for 256
// sequences with a row each, 7.3 for 96 with 54000 rows).
// Every workgroup makes the sums for itself (the lengths come out of L2, which is less than a second launch), and
// writes a slice of the items.
#include "kvd_q8.h"

namespace kvd {
namespace q8 {

constexpr int kMapThreads = 512;

struct MapArgs {
  const int32_t *seq_len, *n_new, *free_blocks, *free_count;
  int32_t *table, *kv_len, *row_start, *row_seq, *row_pos, *counts;
  int4* runs;
  int B, NP, T, R, P, n_free;
};

// Largest i with at[i] <= x, for at[0] = 0 <= x; at ascends.  Of equal entries the last: empty sequences own nothing.
__device__ __forceinline__ int owner(const int* at, int n, int x) {
  int lo = 0;
  for (int hi = n; hi - lo > 1;) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kMapThreads) void map_kernel(MapArgs a) {
  extern __shared__ int lds[];
  int *rows0 = lds, *runs0 = rows0 + a.B, *new0 = runs0 + a.B;
  __shared__ int scan[kMapThreads / kWave + 1];
  const int tid = threadIdx.x, per = (a.B + kMapThreads - 1) / kMapThreads;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  const long long most = (long long)a.NP * a.P;
  int n_rows = 0, n_runs = 0, n_new = 0, bad = 0;
  auto of = [&](int b, int& len, int& n, int& runs, int& fresh) {
    len = a.seq_len[b];
    n = a.n_new[b];
    if (len < 0 || n < 0 || (long long)len + n > most) { bad |= 8; n = 0; len = 0; }
    if (n > a.T) { bad |= 2; n = 0; }            // (the sums stay below 2^30)
    const int end = len + n;
    runs = n > 0 ? (end - 1) / a.P - len / a.P + 1 : 0;
    fresh = (end + a.P - 1) / a.P - (len + a.P - 1) / a.P;
  };
  for (int b = b0; b < b1; ++b) {
    int len, n, runs, fresh;
    of(b, len, n, runs, fresh);
    n_rows += n; n_runs += runs; n_new += fresh;
  }
  int rows, runs, fresh;                         // of the whole step
  int at_row = block_exclusive_scan<kMapThreads>(n_rows, scan, rows);
  int at_run = block_exclusive_scan<kMapThreads>(n_runs, scan, runs);
  int at_new = block_exclusive_scan<kMapThreads>(n_new, scan, fresh);
  const int have = min(max(a.free_count[0], 0), a.n_free);
  if (fresh > have) bad |= 1;
  if (rows > a.T) bad |= 2;
  if (runs > a.R) bad |= 4;
  int why = 0;
#pragma unroll
  for (int bit = 1; bit < 16; bit <<= 1) why |= __syncthreads_or(bad & bit) ? bit : 0;
  const bool first = blockIdx.x == 0;
  for (int b = b0; b < b1; ++b) {
    int len, n, r, f;
    of(b, len, n, r, f);
    rows0[b] = at_row; runs0[b] = at_run; new0[b] = at_new;
    if (first) {
      a.kv_len[b] = why ? a.seq_len[b] : len + n;
      a.row_start[b] = why ? 0 : at_row;
    }
    at_row += n; at_run += r; at_new += f;
  }
  if (why) rows = runs = fresh = 0;
  if (first && tid == 0) {
    a.row_start[a.B] = rows;
    a.counts[0] = rows; a.counts[1] = runs; a.counts[2] = fresh; a.counts[3] = have - fresh; a.counts[4] = why;
  }
  __syncthreads();
  const int t0 = blockIdx.x * kMapThreads + tid, step = gridDim.x * kMapThreads;
  for (int r = t0; r < a.T; r += step) {
    int b = -1, pos = -1;
    if (r < rows) {
      b = owner(rows0, a.B, r);
      pos = a.seq_len[b] + r - rows0[b];
    }
    a.row_seq[r] = b;
    a.row_pos[r] = pos;
  }
  auto free_block = [&](int i) { return a.free_blocks[have - 1 - i]; };
  for (int i = t0; i < a.R; i += step) {
    int4 run = make_int4(-1, 0, 0, 0);
    if (i < runs) {
      const int b = owner(runs0, a.B, i), len = a.seq_len[b], end = len + a.n_new[b];
      const int page = len / a.P + i - runs0[b], begun = (len + a.P - 1) / a.P;
      const int lo = max(page * a.P, len), hi = min((page + 1) * a.P, end);
      run.x = page >= begun ? free_block(new0[b] + page - begun) : a.table[(size_t)b * a.NP + page];
      run.y = rows0[b] + lo - len;
      run.z = lo - page * a.P;
      run.w = hi - lo;
    }
    a.runs[i] = run;
  }
  for (int i = t0; i < fresh; i += step) {
    const int b = owner(new0, a.B, i), begun = (a.seq_len[b] + a.P - 1) / a.P;
    a.table[(size_t)b * a.NP + begun + i - new0[b]] = free_block(i);
  }
}

}  // namespace q8
}  // namespace kvd

extern "C" int kvd_q8_map(const kvd_q8_rows* r, const int32_t* seq_len, const int32_t* n_new, const int32_t* free_blocks,
                          int32_t n_free, const int32_t* free_count, void* stream) {
  using namespace kvd::q8;
  if (int e = check_rows(r)) return e;
  if (n_free < 0) return KVD_ERR_SHAPE;
  if (!aligned(seq_len, 4) || !aligned(n_new, 4) || !aligned(free_count, 4) || (n_free > 0 && !aligned(free_blocks, 4))) return KVD_ERR_ARG;
  if (!aligned(r->page_table, 4) || !aligned(r->kv_len, 4) || !aligned(r->row_start, 4) || !aligned(r->row_seq, 4) ||
      !aligned(r->row_pos, 4) || !aligned(r->counts, 4) || !aligned(r->runs, 16)) return KVD_ERR_ARG;
  // (the workgroups read the inputs while others write the results)
  if (seq_len == r->kv_len || n_new == r->kv_len || free_count == r->counts + 3) return KVD_ERR_ARG;
  MapArgs a;
  a.seq_len = seq_len; a.n_new = n_new; a.free_blocks = free_blocks; a.free_count = free_count;
  a.table = r->page_table; a.kv_len = r->kv_len; a.row_start = r->row_start; a.row_seq = r->row_seq; a.row_pos = r->row_pos;
  a.counts = r->counts; a.runs = reinterpret_cast<int4*>(r->runs);
  a.B = r->n_seqs; a.NP = r->max_pages; a.T = r->n_rows; a.R = r->max_runs; a.P = r->page_size; a.n_free = n_free;
  const int items = a.T > a.R ? a.T : a.R;
  int blocks = (items + kMapThreads - 1) / kMapThreads;
  if (blocks > 256) blocks = 256;
  hipLaunchKernelGGL(map_kernel, dim3(blocks), dim3(kMapThreads), (size_t)a.B * 12, static_cast<hipStream_t>(stream), a);
  return launched();
}

extern "C" int64_t kvd_q8_workspace_bytes(const kvd_q8_cache* c, const kvd_q8_rows* r, int32_t select) {
  if (int e = kvd::q8::check_cache(c, r)) return e;
  return select ? kvd_q8_select_bytes(c, r) : kvd_q8_attn_bytes(c, r);
}
