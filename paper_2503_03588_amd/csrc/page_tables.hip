// Pages and slots of a serving step's new tokens, from the requests' lengths alone (no host in between): sequence b has
// s = q_start[b] tokens in its pages and gets n = q_len[b] more.  It holds ceil(s / B) pages and needs ceil((s + n) / B);
// the new ones are taken from the list of free pages in the order of the sequences, so a sequence's first new page is
// number sum over the sequences before it of their new pages.  A new page's first token is one of the n (its block starts at
// s or later), so the thread of that token enters it into the table, and every token's slot is page * B + offset.
//
// Bound by latency: a few KB are read and written (3.1 us for 128 sequences of one token, 4.3 for 32 of up to 2048).
// One launch: a workgroup forms the sum over the sequences before its own by itself (two words each, from L2) instead of
// waiting for another workgroup's.
#include "common.h"
#include "overlap.h"

namespace {

constexpr int THREADS = 256;
constexpr int CHUNK_ROWS = 1024;         // rows of a workgroup where one sequence has a workgroup, or several

struct pt_params {
  const int32_t* q_start; const int32_t* q_len; const int32_t* free_pages;
  int32_t* table; int32_t* slots; int32_t* kv_len; int32_t* n_taken;
  int32_t batch, q_rows, n_free, n_pages, B, stride, capacity;
  int32_t seqs_shift;                    // 2^seqs_shift sequences in a workgroup
  int32_t n_chunks;                      // workgroups of a sequence (1 where a workgroup has several sequences)
};

struct pt_seq { int32_t s, n, held, fresh; };
__device__ __forceinline__ pt_seq pt_seq_of(const pt_params& p, int b) {
  pt_seq q;
  int32_t s = p.q_start[b], n = p.q_len[b];
  s = s < 0 ? 0 : (s > p.capacity ? p.capacity : s);
  n = n < 0 ? 0 : (n > p.q_rows ? p.q_rows : n);
  if (n > p.capacity - s) n = p.capacity - s;
  const unsigned B = (unsigned)p.B;      // (s + n + B - 1 stays below 2^32: both are below 2^31)
  q.s = s; q.n = n;
  q.held = (int32_t)(((unsigned)s + B - 1) / B);
  q.fresh = (int32_t)(((unsigned)s + (unsigned)n + B - 1) / B) - q.held;
  return q;
}

__global__ __launch_bounds__(THREADS) void pa_page_tables_kernel(pt_params p) {
  __shared__ int64_t s_sum[THREADS / 64];
  __shared__ int32_t s_scan[2][THREADS];
  __shared__ pt_seq s_seq[THREADS];
  const int t = threadIdx.x, n_seqs = 1 << p.seqs_shift;
  const int group = blockIdx.x / p.n_chunks, chunk = blockIdx.x % p.n_chunks;
  const int first = group << p.seqs_shift;

  // ---- new pages of the sequences before this workgroup's ----
  int64_t before = 0;
  for (int b = t; b < first; b += THREADS) before += pt_seq_of(p, b).fresh;
  for (int d = 32; d > 0; d >>= 1) before += __shfl_xor(before, d);
  if ((t & 63) == 0) s_sum[t >> 6] = before;

  // ---- and of its own ones: an exclusive sum ----
  int32_t mine = 0;
  if (t < n_seqs) {
    pt_seq q = {0, 0, 0, 0};
    if (first + t < p.batch) q = pt_seq_of(p, first + t);
    s_seq[t] = q;
    mine = q.fresh;
    if (chunk == 0 && first + t < p.batch) p.kv_len[first + t] = q.s + q.n;
  }
  s_scan[0][t] = mine;
  __syncthreads();
  int side = 0;
  for (int d = 1; d < n_seqs; d <<= 1) {
    s_scan[side ^ 1][t] = s_scan[side][t] + (t >= d ? s_scan[side][t - d] : 0);
    side ^= 1;
    __syncthreads();
  }
  int64_t base = 0;
  for (int w = 0; w < THREADS / 64; ++w) base += s_sum[w];
  if (t == 0 && chunk == 0 && first + n_seqs >= p.batch) {
    const int64_t all = base + s_scan[side][n_seqs - 1];
    *p.n_taken = (int32_t)(all < 0x7fffffff ? all : 0x7fffffff);
  }

  // ---- rows: 256 / n_seqs threads for a sequence ----
  const int per_shift = 8 - p.seqs_shift;
  const int i = t >> per_shift, b = first + i;
  if (b >= p.batch) return;
  const pt_seq q = s_seq[i];
  base += s_scan[side][i] - q.fresh;
  const int64_t row_end = (int64_t)(chunk + 1) * CHUNK_ROWS;
  const int r_end = p.n_chunks > 1 && row_end < p.q_rows ? (int)row_end : p.q_rows;
  int32_t* table = p.table + (int64_t)b * p.stride;
  int32_t* slots = p.slots + (int64_t)b * p.q_rows;
  for (int64_t r = (int64_t)chunk * CHUNK_ROWS + (t & ((1 << per_shift) - 1)); r < r_end; r += 1 << per_shift) {
    int32_t slot = -1;
    if (r < q.n) {
      const unsigned pos = (unsigned)q.s + (unsigned)r, blk = pos / (unsigned)p.B, off = pos - blk * (unsigned)p.B;
      int32_t page;
      if ((int32_t)blk >= q.held) {
        const int64_t which = base + ((int32_t)blk - q.held);
        page = which < p.n_free ? p.free_pages[which] : -1;
        if (off == 0) table[blk] = page;
      } else {
        page = table[blk];               // the last held page, partly filled: this launch writes no entry before q.held
      }
      if (page >= 0 && page < p.n_pages) slot = page * p.B + (int32_t)off;
    }
    slots[r] = slot;
  }
}

}  // namespace

extern "C" int powattn_page_tables(const powattn_pattern* pattern, const int32_t* d_q_start, const int32_t* d_q_len, int32_t batch,
                                   int64_t q_rows, const int32_t* d_free_pages, int32_t n_free, int64_t n_pages,
                                   int32_t* d_block_table, int32_t table_stride, int32_t* d_slots, int32_t* d_kv_len,
                                   int32_t* d_n_taken, void* hip_stream) {
  int st = pa_check_pattern(pattern);
  if (st != POWATTN_OK) return st;
  if (!d_q_start || !d_q_len || !d_block_table || !d_slots || !d_kv_len || !d_n_taken) return POWATTN_INVALID_ARG;
  if (batch < 1 || q_rows < 1 || n_free < 0 || n_pages < 1 || table_stride < 1) return POWATTN_INVALID_ARG;
  if (n_free > 0 && !d_free_pages) return POWATTN_INVALID_ARG;
  const int64_t capacity = (int64_t)table_stride * pattern->block;
  if (q_rows > capacity) return POWATTN_INVALID_ARG;
  if (capacity > 0x7fffffff || n_pages > 0x7fffffff / pattern->block) return POWATTN_UNSUPPORTED;   // slots and positions are 32-bit numbers
  // (every workgroup reads the lengths of the sequences before its own, so an output in their place would change them under it)
  const struct { const void* p; int64_t bytes; } mem[] = {
      {d_block_table, 4 * (int64_t)batch * table_stride}, {d_slots, 4 * (int64_t)batch * q_rows}, {d_kv_len, 4 * (int64_t)batch}, {d_n_taken, 4},
      {d_q_start, 4 * (int64_t)batch}, {d_q_len, 4 * (int64_t)batch}, {d_free_pages, 4 * (int64_t)n_free}};
  for (int o = 0; o < 4; ++o)
    for (int i = o + 1; i < (n_free > 0 ? 7 : 6); ++i)
      if (pa_ranges_meet(mem[o].p, mem[o].bytes, mem[i].p, mem[i].bytes)) return POWATTN_INVALID_ARG;
  pt_params p;
  p.q_start = d_q_start; p.q_len = d_q_len; p.free_pages = d_free_pages;
  p.table = d_block_table; p.slots = d_slots; p.kv_len = d_kv_len; p.n_taken = d_n_taken;
  p.batch = batch; p.q_rows = (int32_t)q_rows; p.n_free = n_free; p.n_pages = (int32_t)n_pages;
  p.B = pattern->block; p.stride = table_stride; p.capacity = (int32_t)capacity;
  // sequences of a workgroup: as many as have a thread for every row; one from 129 rows on
  p.seqs_shift = 8;
  while (p.seqs_shift > 0 && (q_rows << p.seqs_shift) > THREADS) --p.seqs_shift;
  p.n_chunks = p.seqs_shift > 0 ? 1 : (int32_t)((q_rows + CHUNK_ROWS - 1) / CHUNK_ROWS);
  const int64_t groups = ((int64_t)batch + (1 << p.seqs_shift) - 1) >> p.seqs_shift;
  const int64_t wgs = groups * p.n_chunks;
  if (wgs > 0xffffffffLL / THREADS) return POWATTN_UNSUPPORTED;      // a launch has fewer than 2^32 threads
  hipLaunchKernelGGL(pa_page_tables_kernel, dim3((uint32_t)wgs), dim3(THREADS), 0, (hipStream_t)hip_stream, p);
  return pa_note_hip(hipGetLastError());
}
