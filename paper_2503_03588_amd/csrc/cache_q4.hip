// Rows of keys and values into the 4-bit cache and out of it (format: q4.h).
//
// Both move bytes and nothing else: a lane has 8 components, 16 bytes in bf16 and 4 in the cache, four lanes share a scale,
// and a wavefront takes consecutive tokens of one head, so that its pieces of a page are one contiguous stretch.
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
  int32_t n_tokens, rows, hkv, B, n_slots;
};

template <bool VEC>
__device__ __forceinline__ u32x4 q4_load8(const uint16_t* p) {
  if constexpr (VEC) return *reinterpret_cast<const u32x4*>(p);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  return r;
}

// D: head_dim; TOK: tokens of a lane, a wavefront's worth apart, all of them requested before any is used
template <int D, int TOK, bool VEC>
__global__ __launch_bounds__(THREADS) void pa_cache_store_q4_kernel(store_params p) {
  constexpr int LPR = D / 8, STEP = THREADS / LPR;          // lanes of a row, rows side by side
  const int lane = threadIdx.x % LPR, kv = blockIdx.z, h = blockIdx.y;
  const int t0 = blockIdx.x * (STEP * TOK) + threadIdx.x / LPR;
  const q4_rows in = p.in[kv];
  int32_t slot[TOK];
  u32x4 x[TOK];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const int t = t0 + i * STEP;
    slot[i] = t < p.n_tokens ? p.slots[t] : -1;
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    x[i] = u32x4{0, 0, 0, 0};
    if (slot[i] < 0 || slot[i] >= p.n_slots) continue;      // rows without a slot are not read
    const unsigned t = t0 + i * STEP, b = t / (unsigned)p.rows, r = t - b * (unsigned)p.rows;
    x[i] = q4_load8<VEC>(in.p + b * in.sb + h * in.sh + r * in.sr + 8 * lane);
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = (x[i][e] & 0x7fffu) << 16, hi = x[i][e] & 0x7fff0000u;      // magnitudes order like their bits
      amax = max(amax, max(lo, hi));
    }
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    if (slot[i] < 0 || slot[i] >= p.n_slots) continue;
    const uint32_t code = q4_scale_code(amax);
    uint32_t word = 0;
    if (code != 255u) {
      const float scale = q4_scale(code);
      word = q4_shrink<0>(word, x[i][0], scale);
      word = q4_shrink<1>(word, x[i][1], scale);
      word = q4_shrink<2>(word, x[i][2], scale);
      word = q4_shrink<3>(word, x[i][3], scale);
    }
    const unsigned page = (unsigned)slot[i] / (unsigned)p.B, off = (unsigned)slot[i] - page * (unsigned)p.B;
    const int64_t at = (int64_t)page * p.hkv + h;
    *reinterpret_cast<uint32_t*>(p.pages[kv] + (at * p.B + off) * (D / 2) + 4 * lane) = word;
    if ((lane & 3) == 0) p.scales[kv][(at * (D / 32) + (lane >> 2)) * p.B + off] = (uint8_t)code;
  }
}

struct load_params {
  const uint8_t* pages[2]; const uint8_t* scales[2];
  uint16_t* out[2];                       // [batch, heads, rows, head_dim]
  const int32_t* table; const int32_t* start; const int32_t* length;
  int32_t n_tokens, rows, hkv, B, stride, last_page, capacity;
};

template <int D, int TOK>
__global__ __launch_bounds__(THREADS) void pa_cache_load_q4_kernel(load_params p) {
  constexpr int LPR = D / 8, STEP = THREADS / LPR;
  const int lane = threadIdx.x % LPR, kv = blockIdx.z, h = blockIdx.y;
  const int t0 = blockIdx.x * (STEP * TOK) + threadIdx.x / LPR;
  uint32_t word[TOK], code[TOK];
  int64_t to[TOK];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const unsigned t = t0 + i * STEP;
    to[i] = -1;
    word[i] = code[i] = 0;
    if (t >= (unsigned)p.n_tokens) continue;
    const unsigned b = t / (unsigned)p.rows, r = t - b * (unsigned)p.rows;
    int32_t s = p.start ? p.start[b] : 0, n = p.length ? p.length[b] : p.rows;
    s = s < 0 ? 0 : (s > p.capacity ? p.capacity : s);
    if (n > p.capacity - s) n = p.capacity - s;
    if ((int32_t)r >= n) continue;
    const unsigned pos = (unsigned)s + r, blk = pos / (unsigned)p.B, off = pos - blk * (unsigned)p.B;
    int page = p.table[(int64_t)b * p.stride + blk];
    page = page < 0 ? 0 : (page > p.last_page ? p.last_page : page);     // a bad table gives wrong numbers, no stray access
    const int64_t at = (int64_t)page * p.hkv + h;
    word[i] = *reinterpret_cast<const uint32_t*>(p.pages[kv] + (at * p.B + off) * (D / 2) + 4 * lane);
    code[i] = p.scales[kv][(at * (D / 32) + (lane >> 2)) * p.B + off];
    to[i] = (((int64_t)b * p.hkv + h) * p.rows + r) * D + 8 * lane;
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    if (to[i] < 0) continue;
    const float scale = q4_scale(code[i]);
    const u32x4 x = {q4_expand<0>(word[i], scale), q4_expand<1>(word[i], scale), q4_expand<2>(word[i], scale), q4_expand<3>(word[i], scale)};
    *reinterpret_cast<u32x4*>(p.out[kv] + to[i]) = x;
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

// Tokens of a lane: four where that leaves eight wavefronts for every compute unit, else one.
int tokens_of_a_lane(int64_t n_tokens, int32_t hkv, int32_t head_dim) {
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  return n_tokens * hkv * 2 * (head_dim / 8) >= (int64_t)n_cu * 4 * 8 * 64 ? 4 : 1;
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
  if (((uintptr_t)k_pages | (uintptr_t)v_pages) & 15u) return POWATTN_INVALID_ARG;
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
  const int tok = tokens_of_a_lane(p.n_tokens, n_kv_heads, head_dim), step = THREADS / (head_dim / 8);
  const dim3 grid((uint32_t)((p.n_tokens + (int64_t)step * tok - 1) / ((int64_t)step * tok)), (uint32_t)n_kv_heads, 2);
  if ((int64_t)grid.x * grid.y * 2 > 0xffffffffLL / THREADS) return POWATTN_UNSUPPORTED;   // a launch has fewer than 2^32 threads
  hipStream_t stream = (hipStream_t)hip_stream;
#define STORE(D, TOK, VEC) hipLaunchKernelGGL((pa_cache_store_q4_kernel<D, TOK, VEC>), grid, dim3(THREADS), 0, stream, p)
  if (head_dim == 128) {
    if (tok == 4) { if (vec) STORE(128, 4, true); else STORE(128, 4, false); }
    else { if (vec) STORE(128, 1, true); else STORE(128, 1, false); }
  } else {
    if (tok == 4) { if (vec) STORE(64, 4, true); else STORE(64, 4, false); }
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
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k | (uintptr_t)v) & 15u) return POWATTN_INVALID_ARG;
  const int64_t capacity = (int64_t)table_stride * pattern->block;
  if (capacity > 0x7fffffff) return POWATTN_UNSUPPORTED;
  load_params p;
  p.pages[0] = (const uint8_t*)k_pages; p.pages[1] = (const uint8_t*)v_pages;
  p.scales[0] = (const uint8_t*)k_scales; p.scales[1] = (const uint8_t*)v_scales;
  p.out[0] = (uint16_t*)k; p.out[1] = (uint16_t*)v;
  p.table = d_block_table; p.start = d_start; p.length = d_length;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.hkv = n_kv_heads; p.B = pattern->block;
  p.stride = table_stride; p.last_page = (int32_t)n_pages - 1; p.capacity = (int32_t)capacity;
  const int tok = tokens_of_a_lane(p.n_tokens, n_kv_heads, head_dim), step = THREADS / (head_dim / 8);
  const dim3 grid((uint32_t)((p.n_tokens + (int64_t)step * tok - 1) / ((int64_t)step * tok)), (uint32_t)n_kv_heads, 2);
  if ((int64_t)grid.x * grid.y * 2 > 0xffffffffLL / THREADS) return POWATTN_UNSUPPORTED;
  hipStream_t stream = (hipStream_t)hip_stream;
#define LOAD(D, TOK) hipLaunchKernelGGL((pa_cache_load_q4_kernel<D, TOK>), grid, dim3(THREADS), 0, stream, p)
  if (head_dim == 128) { if (tok == 4) LOAD(128, 4); else LOAD(128, 1); }
  else { if (tok == 4) LOAD(64, 4); else LOAD(64, 1); }
#undef LOAD
  return pa_note_hip(hipGetLastError());
}
