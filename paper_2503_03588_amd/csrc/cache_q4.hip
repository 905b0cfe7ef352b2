// Rows of keys and values into the 4-bit cache and out of it (format: q4.h).
//
// Both move bytes and nothing else.  A lane has 8 components, 16 bytes in bf16 and 4 in the cache, four lanes share a scale.
// Where there are rows enough, a lane has four consecutive ones: they mostly lie side by side in a page, and their scales
// are one word then.  A workgroup looks its rows' slots (pages) up once and walks through heads, keys and values
// together; the next head's rows are requested before the current one's are converted.  With few rows a lane has one, of the keys or
// of the values.
#include "common.h"
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
// Four consecutive rows whose slots (positions) follow one another from a multiple of four on, which four rows of a page do
template <int TOK>
__device__ __forceinline__ bool q4_side_by_side(const int32_t (&slot)[TOK]) {
  if constexpr (TOK != 4) return false;
  else return slot[0] >= 0 && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 && slot[3] == slot[0] + 3;
}

// D: head_dim; TOK: consecutive rows of a lane, of keys and of values (one: blockIdx.z says of which)
template <int D, int TOK, bool VEC>
__global__ __launch_bounds__(THREADS) void pa_cache_store_q4_kernel(store_params p) {
  constexpr int LPR = D / 8, NKV = TOK == 1 ? 1 : 2;        // lanes of a row
  const int lane = threadIdx.x % LPR, kv0 = NKV == 1 ? blockIdx.z : 0;
  const int64_t t0 = ((int64_t)blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR) * TOK;
  const int h0 = blockIdx.y * p.per_chunk, h1 = min(h0 + p.per_chunk, p.hkv);
  int32_t slot[TOK];
  const uint16_t* from[NKV][TOK];
  int64_t page[TOK]; int32_t off[TOK];
  bool any = false;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    slot[i] = t0 + i < p.n_tokens ? p.slots[t0 + i] : -1;
    if (slot[i] >= p.n_slots) slot[i] = -1;                 // rows without a slot are not read
    any = any || slot[i] >= 0;
  }
  if (!any) return;                                         // (the lanes of a row stay together)
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const unsigned t = (unsigned)(t0 + i), b = t / (unsigned)p.rows, r = t - b * (unsigned)p.rows;
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv) from[kv][i] = p.in[kv0 + kv].p + b * p.in[kv0 + kv].sb + r * p.in[kv0 + kv].sr + 8 * lane;
    const unsigned pg = (unsigned)max(slot[i], 0) / (unsigned)p.B;
    page[i] = (int64_t)pg * p.hkv;
    off[i] = max(slot[i], 0) - (int)pg * p.B;
  }
  const bool together = q4_side_by_side<TOK>(slot);         // (a block is a multiple of 64 rows: they are in one page)
  u32x4 x[NKV][TOK], next[NKV][TOK];
  auto request = [&](u32x4 (&y)[NKV][TOK], int h) {
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv)
#pragma unroll
      for (int i = 0; i < TOK; ++i) {
        y[kv][i] = u32x4{0, 0, 0, 0};
        if (slot[i] >= 0) y[kv][i] = q4_load8<VEC>(from[kv][i] + h * p.in[kv0 + kv].sh);
      }
  };
  request(x, h0);
  for (int h = h0; h < h1; ++h) {
    if (h + 1 < h1) request(next, h + 1);
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv) {
      uint32_t codes = 0;
#pragma unroll
      for (int i = 0; i < TOK; ++i) {
        const u32x4 y = x[kv][i];
        uint32_t amax = 0;                                  // magnitudes order like their bits
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = max(amax, max((y[e] & 0x7fffu) << 16, y[e] & 0x7fff0000u));
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
        const uint32_t code = q4_scale_code(amax);
        uint32_t word = 0;
        if (code != 255u) {
          const float scale = q4_scale(code);
          word = q4_shrink<0>(word, y[0], scale);
          word = q4_shrink<1>(word, y[1], scale);
          word = q4_shrink<2>(word, y[2], scale);
          word = q4_shrink<3>(word, y[3], scale);
        }
        codes |= code << (8 * i);
        if (slot[i] < 0) continue;
        const int64_t at = page[i] + h;
        *reinterpret_cast<uint32_t*>(p.pages[kv0 + kv] + (at * p.B + off[i]) * (D / 2) + 4 * lane) = word;
        if ((lane & 3) == 0 && !together) p.scales[kv0 + kv][(at * (D / 32) + (lane >> 2)) * p.B + off[i]] = (uint8_t)code;
      }
      if ((lane & 3) == 0 && together)
        *reinterpret_cast<uint32_t*>(p.scales[kv0 + kv] + ((page[0] + h) * (D / 32) + (lane >> 2)) * p.B + off[0]) = codes;
    }
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv)
#pragma unroll
      for (int i = 0; i < TOK; ++i) x[kv][i] = next[kv][i];
  }
}

struct load_params {
  const uint8_t* pages[2]; const uint8_t* scales[2];
  uint16_t* out[2];                       // [batch, heads, rows, head_dim]
  const int32_t* table; const int32_t* start; const int32_t* length;
  int32_t n_tokens, rows, hkv, B, stride, last_page, capacity, per_chunk;
};

template <int D, int TOK>
__global__ __launch_bounds__(THREADS) void pa_cache_load_q4_kernel(load_params p) {
  constexpr int LPR = D / 8, NKV = TOK == 1 ? 1 : 2;
  const int lane = threadIdx.x % LPR, kv0 = NKV == 1 ? blockIdx.z : 0;
  const int64_t t0 = ((int64_t)blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR) * TOK;
  const int h0 = blockIdx.y * p.per_chunk, h1 = min(h0 + p.per_chunk, p.hkv);
  int64_t page[TOK], to[TOK];
  int32_t off[TOK], where[TOK];
  bool any = false;
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    where[i] = -1;
    page[i] = to[i] = off[i] = 0;
    if (t0 + i >= p.n_tokens) continue;
    const unsigned t = (unsigned)(t0 + i), b = t / (unsigned)p.rows, r = t - b * (unsigned)p.rows;
    int32_t s = p.start ? p.start[b] : 0, n = p.length ? p.length[b] : p.rows;
    s = s < 0 ? 0 : (s > p.capacity ? p.capacity : s);
    if (n > p.capacity - s) n = p.capacity - s;
    if ((int32_t)r >= n) continue;
    const unsigned pos = (unsigned)s + r, blk = pos / (unsigned)p.B;
    int pg = p.table[(int64_t)b * p.stride + blk];
    pg = pg < 0 ? 0 : (pg > p.last_page ? p.last_page : pg);             // a bad table gives wrong numbers, no stray access
    page[i] = (int64_t)pg * p.hkv;
    off[i] = (int32_t)(pos - blk * (unsigned)p.B);
    where[i] = pg * p.B + off[i];
    to[i] = ((int64_t)b * p.hkv * p.rows + r) * D + 8 * lane;
    any = true;
  }
  if (!any) return;
  const bool together = q4_side_by_side<TOK>(where);
  uint32_t word[NKV][TOK], code[NKV][TOK], next_word[NKV][TOK], next_code[NKV][TOK];
  auto request = [&](uint32_t (&w)[NKV][TOK], uint32_t (&c)[NKV][TOK], int h) {
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv) {
      if (together) c[kv][0] = *reinterpret_cast<const uint32_t*>(p.scales[kv0 + kv] + ((page[0] + h) * (D / 32) + (lane >> 2)) * p.B + off[0]);
#pragma unroll
      for (int i = 0; i < TOK; ++i) {
        if (where[i] < 0) continue;
        const int64_t at = page[i] + h;
        w[kv][i] = *reinterpret_cast<const uint32_t*>(p.pages[kv0 + kv] + (at * p.B + off[i]) * (D / 2) + 4 * lane);
        if (!together) c[kv][i] = p.scales[kv0 + kv][(at * (D / 32) + (lane >> 2)) * p.B + off[i]];
      }
    }
  };
  request(word, code, h0);
  for (int h = h0; h < h1; ++h) {
    if (h + 1 < h1) request(next_word, next_code, h + 1);
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv)
#pragma unroll
      for (int i = 0; i < TOK; ++i) {
        if (where[i] < 0) continue;
        const float scale = q4_scale(together ? code[kv][0] >> (8 * i) & 255u : code[kv][i]);
        const uint32_t w = word[kv][i];
        const u32x4 x = {q4_expand<0>(w, scale), q4_expand<1>(w, scale), q4_expand<2>(w, scale), q4_expand<3>(w, scale)};
        u32x4* to_row = reinterpret_cast<u32x4*>(p.out[kv0 + kv] + to[i] + (int64_t)h * p.rows * D);
        if constexpr (TOK == 4) __builtin_nontemporal_store(x, to_row);      // (us, 32 pieces of up to 2048 rows: 45 -> 40)
        else *to_row = x;
      }
#pragma unroll
    for (int kv = 0; kv < NKV; ++kv)
#pragma unroll
      for (int i = 0; i < TOK; ++i) { word[kv][i] = next_word[kv][i]; code[kv][i] = next_code[kv][i]; }
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

// The launch: four rows of a lane where that leaves a workgroup for every compute unit, else one; as many heads of a workgroup as
// leave eight workgroups for every compute unit.
struct q4_launch { int tok; int32_t per_chunk; dim3 grid; };
bool launch_of(q4_launch& l, int64_t n_tokens, int32_t hkv, int32_t head_dim) {
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  const int64_t side = THREADS / (head_dim / 8);
  l.tok = n_tokens * hkv >= 4 * side * n_cu ? 4 : 1;
  const int64_t groups = (n_tokens + side * l.tok - 1) / (side * l.tok);
  int64_t chunks = (8 * (int64_t)n_cu + groups - 1) / groups;
  if (chunks > hkv) chunks = hkv;
  l.per_chunk = (int32_t)((hkv + chunks - 1) / chunks);
  l.grid = dim3((uint32_t)groups, (uint32_t)((hkv + l.per_chunk - 1) / l.per_chunk), l.tok == 1 ? 2 : 1);
  return (int64_t)l.grid.x * l.grid.y * l.grid.z <= 0xffffffffLL / THREADS;      // a launch has fewer than 2^32 threads
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
  q4_launch l;
  if (!launch_of(l, p.n_tokens, n_kv_heads, head_dim)) return POWATTN_UNSUPPORTED;
  p.per_chunk = l.per_chunk;
  hipStream_t stream = (hipStream_t)hip_stream;
#define STORE(D, TOK, VEC) hipLaunchKernelGGL((pa_cache_store_q4_kernel<D, TOK, VEC>), l.grid, dim3(THREADS), 0, stream, p)
  if (head_dim == 128) {
    if (l.tok == 4) { if (vec) STORE(128, 4, true); else STORE(128, 4, false); }
    else { if (vec) STORE(128, 1, true); else STORE(128, 1, false); }
  } else {
    if (l.tok == 4) { if (vec) STORE(64, 4, true); else STORE(64, 4, false); }
    else { if (vec) STORE(64, 1, true); else STORE(64, 1, false); }
  }
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
  load_params p;
  p.pages[0] = (const uint8_t*)k_pages; p.pages[1] = (const uint8_t*)v_pages;
  p.scales[0] = (const uint8_t*)k_scales; p.scales[1] = (const uint8_t*)v_scales;
  p.out[0] = (uint16_t*)k; p.out[1] = (uint16_t*)v;
  p.table = d_block_table; p.start = d_start; p.length = d_length;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.hkv = n_kv_heads; p.B = pattern->block;
  p.stride = table_stride; p.last_page = (int32_t)n_pages - 1; p.capacity = (int32_t)capacity;
  q4_launch l;
  if (!launch_of(l, p.n_tokens, n_kv_heads, head_dim)) return POWATTN_UNSUPPORTED;
  p.per_chunk = l.per_chunk;
  hipStream_t stream = (hipStream_t)hip_stream;
#define LOAD(D, TOK) hipLaunchKernelGGL((pa_cache_load_q4_kernel<D, TOK>), l.grid, dim3(THREADS), 0, stream, p)
  if (head_dim == 128) { if (l.tok == 4) LOAD(128, 4); else LOAD(128, 1); }
  else { if (l.tok == 4) LOAD(64, 4); else LOAD(64, 1); }
#undef LOAD
  return pa_note_hip(hipGetLastError());
}
