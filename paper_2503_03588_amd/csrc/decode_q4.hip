// Split-K decode over a paged cache held in 4 bits (format: q4.h): the step of decode.hip with pages of 4-bit keys and values.
//
// A step reads 2 * (head_dim / 2 + head_dim / 32) bytes per attended token and KV head, 0.27 of the bf16 step's.  Values are
// expanded to bf16 in registers, exactly (a 4-bit value times a power of two is a bf16 number), and multiplied on the matrix
// cores: S^T = K q^T, O^T += V^T P^T with v_mfma_f32_16x16x32_bf16.
//  * A chunk is 64 tokens of a block.  Token 4i + T of it is row i of tile T (T = 0..3) of S^T, so that
//    - a lane's 16 bytes of K are one scale's 32 components of a token (head_dim 64: 8 bytes, half a group), and its scales
//      of the four tiles are the four bytes of one word;
//    - lane (g, q4)'s scores are those of tokens 16 q4 .. 16 q4 + 15 for query head g, and the V of these tokens is what it
//      has to supply for the second product: it reads head_dim / 16 components of each of the 16 tokens, whose scales are the
//      16 bytes of one load; pairs of tokens are brought together by byte permutes.
//  * P is multiplied in two parts, bf16 each, so that its rounding is 2^-17 instead of 2^-9 (which would add as much again to
//    the error of the bf16 output): up to 8 query heads take columns 0..7 of the 16, and 8..15 hold the rest of the same
//    heads' P; with more heads there is a second product.
#include <math.h>
#include "decode.h"
#include "q4.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct q4_params {
  dec_params d;                          // (k, v, packets, gen are not used)
  const uint8_t* k; const uint8_t* v; const uint8_t* ks; const uint8_t* vs;
};

// A chunk's registers.  Rows behind the last attended token are not read (a buffer load answers zeros).
template <int D> struct q4_chunk;
template <> struct q4_chunk<128> { u32x4 k[4]; uint32_t v[16]; uint32_t ks; u32x4 vs; };
template <> struct q4_chunk<64> { u32x2 k[4]; uint32_t v[16]; uint32_t ks; u32x4 vs; };

template <int D>
__device__ __forceinline__ void q4_issue(q4_chunk<D>& c, const q4_params& p, int page, int kvh, int sub, int n_tok, int g, int q4) {
  constexpr int ROW = D / 2;
  page = page < 0 ? 0 : (page > p.d.last_page ? p.d.last_page : page);
  const int64_t at = (int64_t)page * p.d.hkv + kvh;
  const int64_t data = (at * p.d.B + sub * CH) * ROW, scale = at * (D / 32) * p.d.B + sub * CH;
  const dec_buf kb = dec_buffer(p.k + data, n_tok * ROW), vb = dec_buffer(p.v + data, n_tok * ROW);
  const int scales = (D / 32 - 1) * p.d.B + CH;
  const dec_buf ksb = dec_buffer(p.ks + scale, scales), vsb = dec_buffer(p.vs + scale, scales);
  if constexpr (D == 128) {
    c.ks = __builtin_amdgcn_raw_buffer_load_b32(ksb, q4 * p.d.B + 4 * g, 0, 0);
#pragma unroll
    for (int T = 0; T < 4; ++T) c.k[T] = __builtin_amdgcn_raw_buffer_load_b128(kb, 4 * g * ROW + 16 * q4 + T * ROW, 0, 0);
    c.vs = __builtin_amdgcn_raw_buffer_load_b128(vsb, (g >> 2) * p.d.B + 16 * q4, 0, 0);
#pragma unroll
    for (int j = 0; j < 16; ++j) c.v[j] = __builtin_amdgcn_raw_buffer_load_b32(vb, 16 * q4 * ROW + 4 * g + j * ROW, 0, 0);
  } else {
    c.ks = __builtin_amdgcn_raw_buffer_load_b32(ksb, (q4 >> 1) * p.d.B + 4 * g, 0, 0);
#pragma unroll
    for (int T = 0; T < 4; ++T) c.k[T] = __builtin_amdgcn_raw_buffer_load_b64(kb, 4 * g * ROW + 8 * q4 + T * ROW, 0, 0);
    c.vs = __builtin_amdgcn_raw_buffer_load_b128(vsb, (g >> 3) * p.d.B + 16 * q4, 0, 0);
#pragma unroll
    for (int j = 0; j < 16; ++j) c.v[j] = __builtin_amdgcn_raw_buffer_load_b16(vb, 16 * q4 * ROW + 2 * g + j * ROW, 0, 0);
  }
  __builtin_amdgcn_sched_barrier(0);       // every load is under way before the first product
}

__device__ __forceinline__ float q4_scale_of(uint32_t word, int byte) { return q4_scale(word >> (8 * byte) & 255u); }
template <int SEL>
__device__ __forceinline__ void q4_pair(uint32_t& lo, uint32_t& hi, uint32_t a, float sa, uint32_t b, float sb) {
  const uint32_t x = q4_expand<SEL>(a, sa), y = q4_expand<SEL>(b, sb);
  lo = __builtin_amdgcn_perm(y, x, 0x05040100u);     // the even component of both tokens
  hi = __builtin_amdgcn_perm(y, x, 0x07060302u);
}

// One online-softmax update with the chunk.  FIRST: nothing has been accumulated yet.
template <int D, bool WIDE>
__device__ __forceinline__ void q4_consume(q4_chunk<D>& c, const bf16x8 (&qf)[D / 32], int n_tok, float c2, int g, int q4,
                                           float& m_run, float& l_run, f32x4 (&O)[D / 16]) {
  constexpr int NT = D / 16;
  f32x4 S[4];
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    S[T] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float sc = q4_scale_of(c.ks, T);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const uint32_t w = c.k[T][s];
      const u32x4 a = {q4_expand<0>(w, sc), q4_expand<1>(w, sc), q4_expand<2>(w, sc), q4_expand<3>(w, sc)};
      S[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), qf[s], S[T], 0, 0, 0);
    }
  }
  // ---- S[T][r] is token 16 q4 + 4 r + T of this lane's head ----
  if (n_tok < CH) {                        // uniform: the sequence's last chunk
    const int left = n_tok - 16 * q4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int T = 0; T < 4; ++T) S[T][r] = 4 * r + T < left ? S[T][r] : -INFINITY;
      // scales of tokens that are not there: whatever the cache holds, no number must not reach 0 * it
      const int n = left - 4 * r;
      c.vs[r] = n >= 4 ? c.vs[r] : (n <= 0 ? 0u : c.vs[r] & ((1u << (8 * n)) - 1u));
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int T = 0; T < 4; ++T)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      S[T][r] *= c2;
      mx = fmaxf(mx, S[T][r]);
    }
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float m_new = fmaxf(m_run, mx);
  // (-inf only where every score so far is: as an underflow or without a number)
  const float ref = m_new == -INFINITY ? 0.f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(m_run - ref);
  m_run = m_new;
  float rowsum = 0.f;
#pragma unroll
  for (int T = 0; T < 4; ++T)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      S[T][r] = __builtin_amdgcn_exp2f(S[T][r] - ref);
      rowsum += S[T][r];
    }
  l_run = l_run * alpha + rowsum;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) O[t][r] *= alpha;

  // ---- O^T += V^T P^T, 32 tokens at a time: k index 8 q4 + 4 tt + r is token 16 q4 + 4 r + 2 u + tt; row i of tile t is
  // component (head_dim / 16) i + t ----
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    bf16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = S[2 * u + (e >> 2)][e & 3];
      hi[e] = (__bf16)x;
      lo[e] = (__bf16)(x - (float)hi[e]);
    }
    if (!WIDE) hi = g < 8 ? hi : lo;
    uint32_t f[NT][4];                     // f[t][pair]: two tokens' component t
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int r = e & 3, T = 2 * u + (e >> 2);
      const uint32_t a = c.v[4 * r + T], b = c.v[4 * r + 4 + T];
      const float sa = q4_scale_of(c.vs[r], T), sb = q4_scale_of(c.vs[r + 1], T);
      q4_pair<0>(f[0][e / 2], f[1][e / 2], a, sa, b, sb);
      q4_pair<1>(f[2][e / 2], f[3][e / 2], a, sa, b, sb);
      if constexpr (D == 128) {
        q4_pair<2>(f[4][e / 2], f[5][e / 2], a, sa, b, sb);
        q4_pair<3>(f[6][e / 2], f[7][e / 2], a, sa, b, sb);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{f[t][0], f[t][1], f[t][2], f[t][3]});
      O[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi, O[t], 0, 0, 0);
      if (WIDE) O[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo, O[t], 0, 0, 0);
    }
  }
}

// D: head_dim; WIDE: more than 8 query heads on a KV head
template <int D, bool WIDE>
__global__ __launch_bounds__(64 * NW) void pa_decode_q4_kernel(q4_params p) {
  constexpr int NT = D / 16;
  __shared__ float s_m[NW][MAXG], s_l[NW][MAXG];
  extern __shared__ __attribute__((aligned(16))) float s_o[];    // [NW][G][D/32][OROW]
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane & 15, q4 = lane >> 4;
  const int G = p.d.G, head = WIDE ? g : g & 7;

  const int len = p.d.kv_len[b];
  // q^T fragments: k index (q4, e) of step s is component (D / 4) q4 + 8 s + e
  bf16x8 qf[D / 32];
  const dec_buf qb = dec_buffer(p.d.q + ((int64_t)b * p.d.hq + (int64_t)kvh * G) * D, G * 2 * D);
#pragma unroll
  for (int s = 0; s < D / 32; ++s) qf[s] = __builtin_bit_cast(bf16x8, dec_load16(qb, head * 2 * D + (D / 2) * q4, 16 * s));
  const dec_row row = dec_row_of(p.d, len);
  const int n_slots = len > 0 ? row.n_slots : 0;                 // an empty sequence attends nothing

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 O[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) O[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int slot = wave * p.d.splits + split; slot < n_slots; slot += NW * p.d.splits) {
    const dec_place pl = dec_place_of(p.d, row, slot);
    if (pl.n_tok <= 0) break;                                    // chunk of the diagonal block beyond the query: the last ones
    q4_chunk<D> c;
    q4_issue<D>(c, p, dec_page(p.d, b, pl.blk), kvh, pl.sub, pl.n_tok, g, q4);
    q4_consume<D, WIDE>(c, qf, pl.n_tok, p.d.c2, g, q4, m_run, l_run, O);
  }

  // ---- the wavefronts' partials meet in LDS ----
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if (!WIDE) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) O[t][r] += __shfl_xor(O[t][r], 8);
  }
  if (g < G) {
    if (q4 == 0) { s_m[wave][g] = m_run; s_l[wave][g] = l_run; }
    // components (D / 4) q4 + (D / 16) r + t
    const int d0 = (D / 4) * q4;
    f32x4* to = reinterpret_cast<f32x4*>(s_o + dec_o_at<D>(wave, G, g, d0));
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; t += 4) to[(NT / 4) * r + t / 4] = f32x4{O[t][r], O[t + 1][r], O[t + 2][r], O[t + 3][r]};
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * D; e += 64 * NW) {
    const int gg = e / D, d = e % D;
    float M = -INFINITY, L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, s_m[w][gg]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float wt = __builtin_amdgcn_exp2f(s_m[w][gg] - ref);
      L = fmaf(wt, s_l[w][gg], L);
      acc = fmaf(wt, s_o[dec_o_at<D>(w, G, gg, d)], acc);
    }
    const int64_t h = (int64_t)b * p.d.hq + kvh * G + gg;
    if (p.d.splits == 1) {
      p.d.o[h * D + d] = (__bf16)(L == 0.f ? 0.f : acc / L);
      if (p.d.lse && d == 0) p.d.lse[h] = (M + log2f(L)) * 0.69314718055994530942f;
    } else {
      float* part = p.d.partials + (h * p.d.splits + split) * (D + 2);
      part[d] = acc;
      if (d == 0) { part[D] = M; part[D + 1] = L; }
    }
  }
}

// Adds up the splits' partials: one wavefront per (sequence, query head).
template <int D>
__global__ __launch_bounds__(64) void pa_decode_q4_merge_kernel(dec_params p) {
  constexpr int DPL = D / 64;
  const int64_t h = (int64_t)blockIdx.y * p.hq + blockIdx.x;
  const int lane = threadIdx.x;
  const float* part = p.partials + h * p.splits * (D + 2);
  float M = -INFINITY;
  for (int s = 0; s < p.splits; ++s) M = fmaxf(M, part[(int64_t)s * (D + 2) + D]);
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f, acc[DPL] = {};
  for (int s = 0; s < p.splits; ++s) {
    const float* ps = part + (int64_t)s * (D + 2);
    const float wt = __builtin_amdgcn_exp2f(ps[D] - ref);
    L = fmaf(wt, ps[D + 1], L);
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] = fmaf(wt, ps[lane + 64 * e], acc[e]);
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) p.o[h * D + lane + 64 * e] = (__bf16)(L == 0.f ? 0.f : acc[e] / L);
  if (p.lse && lane == 0) p.lse[h] = (M + log2f(L)) * 0.69314718055994530942f;
}

int32_t q4_splits(const powattn_pattern* pattern, int32_t batch, int32_t hkv, int64_t capacity) {
  return pa_decode_splits(pattern, batch, hkv, capacity);
}

template <int D, bool WIDE>
int launch_q4(const q4_params& p, int batch, hipStream_t stream) {
  static std::atomic<unsigned long long> attr_done{0};
  if (int st = pa_allow_dynamic_lds(reinterpret_cast<const void*>(&pa_decode_q4_kernel<D, WIDE>), dec_o_bytes<D>(MAXG), attr_done)) return st;
  const dim3 grid((uint32_t)p.d.splits, (uint32_t)p.d.hkv, (uint32_t)batch);
  hipLaunchKernelGGL((pa_decode_q4_kernel<D, WIDE>), grid, dim3(64 * NW), dec_o_bytes<D>(p.d.G), stream, p);
  if (int st = pa_note_hip(hipGetLastError())) return st;
  if (p.d.splits == 1) return POWATTN_OK;
  hipLaunchKernelGGL((pa_decode_q4_merge_kernel<D>), dim3((uint32_t)p.d.hq, (uint32_t)batch), dim3(64), 0, stream, p.d);
  return pa_note_hip(hipGetLastError());
}

}  // namespace

extern "C" size_t powattn_decode_paged_q4_workspace_bytes(const powattn_pattern* pattern, int32_t batch, int32_t n_q_heads,
                                                          int32_t n_kv_heads, int32_t head_dim, int64_t cache_capacity) {
  if (pa_check_pattern(pattern) != POWATTN_OK) return 0;
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || head_dim < 1 || cache_capacity < 1) return 0;
  if (n_q_heads % n_kv_heads != 0) return 0;
  const int32_t ns = q4_splits(pattern, batch, n_kv_heads, cache_capacity);
  if (ns < 1) return 0;
  const size_t bytes = (size_t)batch * n_q_heads * ns * (size_t)(head_dim + 2) * sizeof(float);
  return (bytes + 255) & ~(size_t)255;
}

extern "C" int powattn_decode_paged_q4(const powattn_pattern* pattern, const void* q, const void* k_pages, const void* v_pages,
                                       const void* k_scales, const void* v_scales, int64_t n_pages,
                                       const int32_t* d_block_table, int32_t table_stride, const int32_t* d_kv_len,
                                       void* o, float* lse, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, int32_t dtype, float softmax_scale,
                                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  int st = pa_check_pattern(pattern);
  if (st != POWATTN_OK) return st;
  if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !d_block_table || !d_kv_len || !o) return POWATTN_INVALID_ARG;
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || head_dim < 1 || n_pages < 1 || table_stride < 1) return POWATTN_INVALID_ARG;
  if (n_q_heads % n_kv_heads != 0) return POWATTN_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return POWATTN_INVALID_ARG;
  if (dtype != POWATTN_BF16) return POWATTN_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return POWATTN_UNSUPPORTED;
  if (pattern->block % 64 != 0 || pattern->block > 1024) return POWATTN_UNSUPPORTED;
  if (pattern->flags & POWATTN_DENSE) return POWATTN_UNSUPPORTED;
  if (n_q_heads / n_kv_heads > MAXG) return POWATTN_UNSUPPORTED;
  if (n_kv_heads > 65535 || batch > 65535) return POWATTN_UNSUPPORTED;
  if (n_pages > 0x7fffffff / pattern->block) return POWATTN_UNSUPPORTED;
  if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_scales | (uintptr_t)v_scales) & 15u) return POWATTN_INVALID_ARG;
  const int64_t capacity = (int64_t)table_stride * pattern->block;
  if (powattn_num_blocks(pattern, capacity) < 0) return POWATTN_INVALID_ARG;
  const size_t need = powattn_decode_paged_q4_workspace_bytes(pattern, batch, n_q_heads, n_kv_heads, head_dim, capacity);
  if (need == 0) return POWATTN_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return POWATTN_WORKSPACE_TOO_SMALL;
  if (((uintptr_t)workspace & 255u) != 0) return POWATTN_INVALID_ARG;

  q4_params p = {};
  p.k = (const uint8_t*)k_pages; p.v = (const uint8_t*)v_pages; p.ks = (const uint8_t*)k_scales; p.vs = (const uint8_t*)v_scales;
  dec_params& d = p.d;
  d.q = (const __bf16*)q; d.kv_len = d_kv_len; d.o = (__bf16*)o; d.lse = lse; d.partials = (float*)workspace;
  d.capacity = capacity; d.len_max = (int32_t)(capacity < 0x7fffffff ? capacity : 0x7fffffff);
  d.B = pattern->block; d.W = pattern->window; d.S = pattern->sink; d.flags = pattern->flags;
  d.hq = n_q_heads; d.hkv = n_kv_heads; d.G = n_q_heads / n_kv_heads; d.subs = pattern->block / CH;
  d.subs_magic = d.subs > 1 ? (uint32_t)(((1ull << 32) + d.subs - 1) / d.subs) : 0u;
  d.splits = q4_splits(pattern, batch, n_kv_heads, capacity);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)head_dim);
  d.c2 = scale * 1.44269504088896340736f;
  d.block_table = d_block_table; d.table_stride = table_stride; d.last_page = (int32_t)n_pages - 1;
  hipStream_t stream = (hipStream_t)hip_stream;
  const bool wide = d.G > 8;
  if (head_dim == 128) return wide ? launch_q4<128, true>(p, batch, stream) : launch_q4<128, false>(p, batch, stream);
  return wide ? launch_q4<64, true>(p, batch, stream) : launch_q4<64, false>(p, batch, stream);
}
