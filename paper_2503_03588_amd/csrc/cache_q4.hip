// Rows of keys and values into the 4-bit cache and out of it (format: q4.h).
//
// Both move bytes and nothing else.  A lane has 8 components, 16 bytes in bf16 and 4 in the cache, four lanes share a scale, and a
// wavefront takes consecutive rows, so that its pieces of a page are one stretch.  A workgroup looks its rows' slots (pages)
// up once and walks through heads; the next head's rows are requested before the current one's are converted.
// 34352 and 37399 rows of 8 heads of 128 in turn: stored in 43.7 us (4.3 TB/s), loaded in 33.7 (5.5); the same 37399 rows again and again: stored
// in 36.6 (5.3); 128 rows 3.0 and 2.8.  Whole contexts, 8 of 16384 tokens, loaded cold: 143 us with the launch (4.7 TB/s).
// (Four consecutive rows of a lane, of keys and values both, whose scales are one word then: stored and loaded, 32 pieces of up to 2048 rows
// 99 / 78 us, 4000 rows of 8 heads 14.1 / 13.6, 1000 10.8 / 6.6, 128 10.4 / 4.8.)
#include "common.h"
#include "overlap.h"
#include "q4.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int THREADS = 256;

struct q4_rows {                          // bf16 rows [batch, heads, rows, head_dim] with any strides (in elements)
  const uint16_t* p; int64_t sb, sh, sr;
};
struct store_params {
  q4_rows in[2];                          // keys, values
  uint8_t* pages[2]; uint8_t* scales[2];
  const int32_t* slots;
  int32_t n_tokens, rows, hkv, B, n_slots, per_chunk;
};

template <bool VEC>
__device__ __forceinline__ u32x4 q4_load8(const uint16_t* p) {
  if constexpr (VEC) return *reinterpret_cast<const u32x4*>(p);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  return r;
}

// D: head_dim; blockIdx.z: keys or values
template <int D, bool VEC>
__global__ __launch_bounds__(THREADS) void pa_cache_store_q4_kernel(store_params p) {
  constexpr int LPR = D / 8;                                // lanes of a row
  const int lane = threadIdx.x % LPR, kv = blockIdx.z;
  const int64_t t = (int64_t)blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR;
  const int h0 = blockIdx.y * p.per_chunk, h1 = min(h0 + p.per_chunk, p.hkv);
  const int32_t slot = t < p.n_tokens ? p.slots[t] : -1;
  if (slot < 0 || slot >= p.n_slots) return;                // rows without a slot are not read (the lanes of a row stay together)
  const unsigned b = (unsigned)t / (unsigned)p.rows, r = (unsigned)t - b * (unsigned)p.rows;
  const unsigned page = (unsigned)slot / (unsigned)p.B, off = (unsigned)slot - page * (unsigned)p.B;
  const uint16_t* from = p.in[kv].p + b * p.in[kv].sb + r * p.in[kv].sr + 8 * lane;
  const int64_t sh = p.in[kv].sh;
  u32x4 x = q4_load8<VEC>(from + h0 * sh), next = x;
  for (int h = h0; h < h1; ++h, x = next) {
    if (h + 1 < h1) next = q4_load8<VEC>(from + (h + 1) * sh);
    uint32_t amax = 0;                                      // magnitudes order like their bits
#pragma unroll
    for (int e = 0; e < 4; ++e) amax = max(amax, max((x[e] & 0x7fffu) << 16, x[e] & 0x7fff0000u));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    const uint32_t code = q4_scale_code(amax);
    uint32_t word = 0;
    if (code != 255u) {
      const float scale = q4_scale(code);
      word = q4_shrink<0>(word, x[0], scale);
      word = q4_shrink<1>(word, x[1], scale);
      word = q4_shrink<2>(word, x[2], scale);
      word = q4_shrink<3>(word, x[3], scale);
    }
    const int64_t at = (int64_t)page * p.hkv + h;
    *reinterpret_cast<uint32_t*>(p.pages[kv] + (at * p.B + off) * (D / 2) + 4 * lane) = word;
    if ((lane & 3) == 0) p.scales[kv][(at * (D / 32) + (lane >> 2)) * p.B + off] = (uint8_t)code;
  }
}

struct load_params {
  const uint8_t* pages[2]; const uint8_t* scales[2];
  uint16_t* out[2];                       // [batch, heads, rows, head_dim]
  const int32_t* table; const int32_t* start; const int32_t* length;
  int32_t n_tokens, rows, hkv, B, stride, last_page, capacity, per_chunk;
};

template <int D>
__global__ __launch_bounds__(THREADS) void pa_cache_load_q4_kernel(load_params p) {
  constexpr int LPR = D / 8;
  const int lane = threadIdx.x % LPR, kv = blockIdx.z;
  const int64_t t = (int64_t)blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR;
  const int h0 = blockIdx.y * p.per_chunk, h1 = min(h0 + p.per_chunk, p.hkv);
  if (t >= p.n_tokens) return;
  const unsigned b = (unsigned)t / (unsigned)p.rows, r = (unsigned)t - b * (unsigned)p.rows;
  int32_t s = p.start ? p.start[b] : 0, n = p.length ? p.length[b] : p.rows;
  s = s < 0 ? 0 : (s > p.capacity ? p.capacity : s);
  if (n > p.capacity - s) n = p.capacity - s;
  if ((int32_t)r >= n) return;
  const unsigned pos = (unsigned)s + r, blk = pos / (unsigned)p.B, off = pos - blk * (unsigned)p.B;
  int page = p.table[(int64_t)b * p.stride + blk];
  page = page < 0 ? 0 : (page > p.last_page ? p.last_page : page);       // a bad table gives wrong numbers, no stray access
  uint16_t* to = p.out[kv] + ((int64_t)b * p.hkv * p.rows + r) * D + 8 * lane;
  uint32_t word, code, next_word = 0, next_code = 0;
  auto request = [&](uint32_t& w, uint32_t& c, int h) {
    const int64_t at = (int64_t)page * p.hkv + h;
    w = *reinterpret_cast<const uint32_t*>(p.pages[kv] + (at * p.B + off) * (D / 2) + 4 * lane);
    c = p.scales[kv][(at * (D / 32) + (lane >> 2)) * p.B + off];
  };
  request(word, code, h0);
  for (int h = h0; h < h1; ++h, word = next_word, code = next_code) {
    if (h + 1 < h1) request(next_word, next_code, h + 1);
    const float scale = q4_scale(code);
    const u32x4 x = {q4_expand<0>(word, scale), q4_expand<1>(word, scale), q4_expand<2>(word, scale), q4_expand<3>(word, scale)};
    // past the caches: stored and loaded, us, 32 pieces of up to 2048 rows 78 / 96 through them, 1000 rows 6.6 / 6.7, 128 rows level
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to + (int64_t)h * p.rows * D));
  }
}

// the limits that both calls share
int check_cache(const powattn_pattern* pattern, int32_t batch, int32_t hkv, int64_t rows, int64_t n_pages, int32_t head_dim, int32_t dtype) {
  if (batch < 1 || hkv < 1 || rows < 1 || n_pages < 1 || head_dim < 1) return POWATTN_INVALID_ARG;
  if (dtype != POWATTN_BF16) return POWATTN_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return POWATTN_UNSUPPORTED;
  if (pattern->block % 64 != 0 || pattern->block > 1024) return POWATTN_UNSUPPORTED;
  if (n_pages > 0x7fffffff / pattern->block) return POWATTN_UNSUPPORTED;                  // slots are 32-bit numbers
  if (hkv > 65535 || rows > 0x7fffffff || (int64_t)batch * rows > 0x7fffffff - 4096) return POWATTN_UNSUPPORTED;
  return POWATTN_OK;
}

// Whether one of the first `n_out` pieces of memory, the outputs, shares bytes with another piece.
struct piece { const void* p; int64_t bytes; };
template <int N>
bool outputs_meet(const piece (&m)[N], int n_out) {
  for (int o = 0; o < n_out; ++o)
    for (int i = o + 1; i < N; ++i)
      if (pa_ranges_meet(m[o].p, m[o].bytes, m[i].p, m[i].bytes)) return true;
  return false;
}
int64_t scale_bytes(int64_t n_pages, int32_t hkv, int32_t block, int32_t head_dim) { return n_pages * hkv * block * (head_dim / 32); }

// As many heads of a workgroup as leave eight workgroups for every compute unit.
bool grid_of(dim3& grid, int32_t& per_chunk, int64_t n_tokens, int32_t hkv, int32_t head_dim) {
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  const int64_t side = THREADS / (head_dim / 8), groups = (n_tokens + side - 1) / side;
  int64_t chunks = (8 * (int64_t)n_cu + groups - 1) / groups;
  if (chunks > hkv) chunks = hkv;
  per_chunk = (int32_t)((hkv + chunks - 1) / chunks);
  grid = dim3((uint32_t)groups, (uint32_t)((hkv + per_chunk - 1) / per_chunk), 2);
  return (int64_t)grid.x * grid.y * 2 <= 0xffffffffLL / THREADS;      // a launch has fewer than 2^32 threads
}

}  // namespace

extern "C" int powattn_cache_store_q4(const powattn_pattern* pattern, const void* k, const int64_t* k_strides, const void* v,
                                      const int64_t* v_strides, const int32_t* d_slots, void* k_pages, void* v_pages,
                                      void* k_scales, void* v_scales, int64_t n_pages, int32_t batch, int32_t n_kv_heads,
                                      int64_t rows, int32_t head_dim, int32_t dtype, void* hip_stream) {
  int st = pa_check_pattern(pattern);
  if (st != POWATTN_OK) return st;
  if (!k || !v || !k_strides || !v_strides || !d_slots || !k_pages || !v_pages || !k_scales || !v_scales) return POWATTN_INVALID_ARG;
  if ((st = check_cache(pattern, batch, n_kv_heads, rows, n_pages, head_dim, dtype)) != POWATTN_OK) return st;
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_scales | (uintptr_t)v_scales) & 15u) return POWATTN_INVALID_ARG;
  if (((uintptr_t)k | (uintptr_t)v) & 1u) return POWATTN_INVALID_ARG;
  const int64_t sb = scale_bytes(n_pages, n_kv_heads, pattern->block, head_dim);
  if (outputs_meet<4>({{k_pages, 16 * sb}, {v_pages, 16 * sb}, {k_scales, sb}, {v_scales, sb}}, 4)) return POWATTN_INVALID_ARG;
  store_params p;
  p.in[0] = {(const uint16_t*)k, k_strides[0], k_strides[1], k_strides[2]};
  p.in[1] = {(const uint16_t*)v, v_strides[0], v_strides[1], v_strides[2]};
  p.pages[0] = (uint8_t*)k_pages; p.pages[1] = (uint8_t*)v_pages;
  p.scales[0] = (uint8_t*)k_scales; p.scales[1] = (uint8_t*)v_scales;
  p.slots = d_slots;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.hkv = n_kv_heads; p.B = pattern->block;
  p.n_slots = (int32_t)(n_pages * pattern->block);
  bool vec = (((uintptr_t)k | (uintptr_t)v) & 15u) == 0;
  for (int i = 0; i < 3; ++i) vec = vec && k_strides[i] % 8 == 0 && v_strides[i] % 8 == 0;
  dim3 grid;
  if (!grid_of(grid, p.per_chunk, p.n_tokens, n_kv_heads, head_dim)) return POWATTN_UNSUPPORTED;
  hipStream_t stream = (hipStream_t)hip_stream;
#define STORE(D, VEC) hipLaunchKernelGGL((pa_cache_store_q4_kernel<D, VEC>), grid, dim3(THREADS), 0, stream, p)
  if (head_dim == 128) { if (vec) STORE(128, true); else STORE(128, false); }
  else { if (vec) STORE(64, true); else STORE(64, false); }
#undef STORE
  return pa_note_hip(hipGetLastError());
}

extern "C" int powattn_cache_load_q4(const powattn_pattern* pattern, const void* k_pages, const void* v_pages, const void* k_scales,
                                     const void* v_scales, int64_t n_pages, const int32_t* d_block_table, int32_t table_stride,
                                     const int32_t* d_start, const int32_t* d_length, void* k, void* v, int32_t batch,
                                     int32_t n_kv_heads, int64_t rows, int32_t head_dim, int32_t dtype, void* hip_stream) {
  int st = pa_check_pattern(pattern);
  if (st != POWATTN_OK) return st;
  if (!k || !v || !d_block_table || !k_pages || !v_pages || !k_scales || !v_scales) return POWATTN_INVALID_ARG;
  if (table_stride < 1) return POWATTN_INVALID_ARG;
  if ((st = check_cache(pattern, batch, n_kv_heads, rows, n_pages, head_dim, dtype)) != POWATTN_OK) return st;
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_scales | (uintptr_t)v_scales | (uintptr_t)k | (uintptr_t)v) & 15u) return POWATTN_INVALID_ARG;
  const int64_t capacity = (int64_t)table_stride * pattern->block;
  if (capacity > 0x7fffffff) return POWATTN_UNSUPPORTED;
  const int64_t sb = scale_bytes(n_pages, n_kv_heads, pattern->block, head_dim), out = 2 * (int64_t)batch * n_kv_heads * rows * head_dim;
  if (outputs_meet<6>({{k, out}, {v, out}, {k_pages, 16 * sb}, {v_pages, 16 * sb}, {k_scales, sb}, {v_scales, sb}}, 2)) return POWATTN_INVALID_ARG;
  load_params p;
  p.pages[0] = (const uint8_t*)k_pages; p.pages[1] = (const uint8_t*)v_pages;
  p.scales[0] = (const uint8_t*)k_scales; p.scales[1] = (const uint8_t*)v_scales;
  p.out[0] = (uint16_t*)k; p.out[1] = (uint16_t*)v;
  p.table = d_block_table; p.start = d_start; p.length = d_length;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.hkv = n_kv_heads; p.B = pattern->block;
  p.stride = table_stride; p.last_page = (int32_t)n_pages - 1; p.capacity = (int32_t)capacity;
  dim3 grid;
  if (!grid_of(grid, p.per_chunk, p.n_tokens, n_kv_heads, head_dim)) return POWATTN_UNSUPPORTED;
  hipStream_t stream = (hipStream_t)hip_stream;
  if (head_dim == 128) hipLaunchKernelGGL((pa_cache_load_q4_kernel<128>), grid, dim3(THREADS), 0, stream, p);
  else hipLaunchKernelGGL((pa_cache_load_q4_kernel<64>), grid, dim3(THREADS), 0, stream, p);
  return pa_note_hip(hipGetLastError());
}
