// Split-K decode over a paged cache held in 4 bits (format: q4.h): the step of decode.hip with pages of 4-bit keys and values.
//
// A step reads 2 * (head_dim / 2 + head_dim / 32) bytes per attended token and KV head, 0.27 of the bf16 step's, so that
// it is bound by latency and by the instructions of expanding the cache rather than by memory.
//  * A chunk is 64 tokens of a block; a wavefront requests all of one before it uses any.  Token 4i + T of it is row i of tile T
//    (T = 0..3) of S^T = K q^T, and lane (g, q4) (g = lane % 16, q4 = lane / 16) then has the scores of tokens
//    16 q4 .. 16 q4 + 15.
//  * Keys are not expanded: v_mfma_scale_f32_16x16x128_f8f6f4 takes 4-bit rows with their scales, which are the bytes of one
//    word for a lane's rows of the four tiles.  The other operand is the query in 8 bits, as the sum of two e4m3 numbers with a power of two each
//    for the row: of bf16's 8 bits each has 4 (sign and one implicit bit apart), so the sum is exact for components down to
//    2^-13 of the row's largest, and off by at most 2^-22 of that below, which is less than the rounding of the
//    sum in fp32.  (Expanding the keys to bf16 instead takes 64 conversions and 8 more products a chunk.)
//  * Values are expanded to bf16, exactly.  The conversion yields two neighbouring components of a token; where the
//    product wants pairs along the tokens, a token counts twice in its sum, once for each component, and P is held with zeros in
//    the other place: O_even and O_odd are different columns.  (Bringing pairs of tokens together by byte permutes: 64 more
//    instructions a chunk, and as many products.)
//  * P is multiplied in two parts, the upper 16 bits of its fp32 number and the upper 16 of what is left: 2^-16 off
//    instead of bf16's 2^-9 (which would add as much again to the error of the bf16 output).  Up to 4 query heads (GM = 4): 16
//    columns are 4 heads x even, odd x the two parts; up to 8 (GM = 8): two products; up to 16: four.
//  * The wavefronts' partial (max, sum, O) meet in LDS.
#include <math.h>
#include <type_traits>
#include "decode.h"
#include "q4.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct q4_params {
  dec_params d;                          // (k, v, packets, gen are not used)
  const uint8_t* k; const uint8_t* v; const uint8_t* ks; const uint8_t* vs;
};

// A chunk's registers.  Rows behind the last attended token are not read (a buffer load answers zeros).
//   k   head_dim 128: 32 components (32 q4 ..) of token 4g + T; head_dim 64: 32 components (32 (q4 % 2) ..) of token
//       4g + 2i + q4 / 2, two tiles in a register, the upper half of the lanes having the odd one
//   ks  the scales of tokens 4g .. 4g + 3 for these components
//   v   head_dim / 16 components of tokens 16 q4 + j;  vs  their 16 scales
template <int D>
struct q4_chunk { u32x4 k[D / 32]; uint32_t v[16]; uint32_t ks; u32x4 vs; };

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
    for (int T = 0; T < 4; ++T) c.k[T] = dec_load16(kb, 4 * g * ROW + 16 * q4, T * ROW);
    c.vs = dec_load16(vsb, (g >> 2) * p.d.B + 16 * q4, 0);
#pragma unroll
    for (int j = 0; j < 16; ++j) c.v[j] = __builtin_amdgcn_raw_buffer_load_b32(vb, 16 * q4 * ROW + 4 * g + j * ROW, 0, 0);
  } else {
    c.ks = __builtin_amdgcn_raw_buffer_load_b32(ksb, (q4 & 1) * p.d.B + 4 * g, 0, 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) c.k[i] = dec_load16(kb, (4 * g + (q4 >> 1)) * ROW + 16 * (q4 & 1), 2 * i * ROW);
    c.vs = dec_load16(vsb, (g >> 3) * p.d.B + 16 * q4, 0);
#pragma unroll
    for (int j = 0; j < 16; ++j) c.v[j] = __builtin_amdgcn_raw_buffer_load_b16(vb, 16 * q4 * ROW + 2 * g + j * ROW, 0, 0);
  }
  __builtin_amdgcn_sched_barrier(0);       // every load is under way before the first product
}

// The query as the sum of two e4m3 rows.  Lane (g, q4) supplies components 16 q4 .. 16 q4 + 15 and, at head_dim 128, 64 + those, of
// its column's head (the product's k index of an 8-bit operand; the scale of 32 components is the same for all).
template <int D>
struct q4_query { uint32_t hi[D / 16], lo[D / 16]; int s_hi, s_lo; };
template <int D>
__device__ __forceinline__ q4_query<D> q4_split_query(const u32x4 (&x)[D / 32]) {
  constexpr int N = D / 16;
  q4_query<D> q;
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 2 * N; ++i) {
    const uint32_t w = x[i / 4][i % 4];
    amax = max(amax, max((w & 0x7fffu) << 16, w & 0x7fff0000u));
  }
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
  // the largest component lands in [2^7, 2^8); what the first part leaves is at most 2^3 and is held 2^5 finer
  const int e = (int)(amax >> 23);
  q.s_hi = e == 255 ? 255 : (e < 12 ? 5 : e - 7);        // (infinities and NaN: no score is a number)
  q.s_lo = e == 255 ? 255 : q.s_hi - 5;
  const float s_hi = q4_scale(q.s_hi), s_lo = q4_scale(q.s_lo);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t w0 = x[i / 2][2 * i % 4], w1 = x[i / 2][2 * i % 4 + 1];
    i16x2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(q4_bf16x2, w0), s_hi, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(q4_bf16x2, w1), s_hi, true);
    q.hi[i] = __builtin_bit_cast(uint32_t, a);
    const f32x2 u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q.hi[i], s_hi, false), v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q.hi[i], s_hi, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, __builtin_bit_cast(float, w0 << 16) - u[0], __builtin_bit_cast(float, w0 & 0xffff0000u) - u[1], s_lo, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, __builtin_bit_cast(float, w1 << 16) - v[0], __builtin_bit_cast(float, w1 & 0xffff0000u) - v[1], s_lo, true);
    q.lo[i] = __builtin_bit_cast(uint32_t, b);
  }
  return q;
}
// S += K tile x the query: 4-bit rows with the scales in byte SEL of `ks`
template <int SEL>
__device__ __forceinline__ f32x4 q4_score(const u32x4& k, int ks, const i32x8& hi, const i32x8& lo, int s_hi, int s_lo, f32x4 S) {
  const i32x8 a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
  S = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, hi, S, 4, 0, SEL, ks, 0, s_hi);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, lo, S, 4, 0, SEL, ks, 0, s_lo);
}

// byte BYTE of a word of scales as the conversions want it: they look at the exponent's bits only, so what else is shifted
// along does not matter (checked for every code)
template <int BYTE>
__device__ __forceinline__ float q4_scale_byte(uint32_t word) {
  return __builtin_bit_cast(float, BYTE == 3 ? word >> 1 : word << (23 - 8 * BYTE));
}

// A lane's place among the columns
template <int GM>
struct q4_column {
  int head; bool odd, rest;              // its head; O_odd or O_even; the second part of P (GM = 16: both and both)
  __device__ __forceinline__ explicit q4_column(int g)
      : head(g & (GM - 1)), odd(GM == 4 ? (g & 4) != 0 : GM == 8 && g >= 8), rest(GM == 4 && g >= 8) {}
};

// One online-softmax update with the chunk.
template <int D, int GM>
__device__ __forceinline__ void q4_consume(q4_chunk<D>& c, const q4_query<D>& q, int n_tok, float c2, int g, int q4,
                                           float& m_run, float& l_run, f32x4 (&O)[GM == 16 ? 2 : 1][D / 32]) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 S[4];
  if constexpr (D == 128) {
    i32x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) { hi[i] = (int)q.hi[i]; lo[i] = (int)q.lo[i]; }
    S[0] = q4_score<0>(c.k[0], (int)c.ks, hi, lo, q.s_hi, q.s_lo, zero);
    S[1] = q4_score<1>(c.k[1], (int)c.ks, hi, lo, q.s_hi, q.s_lo, zero);
    S[2] = q4_score<2>(c.k[2], (int)c.ks, hi, lo, q.s_hi, q.s_lo, zero);
    S[3] = q4_score<3>(c.k[3], (int)c.ks, hi, lo, q.s_hi, q.s_lo, zero);
  } else {
    // a register has two tokens' rows; the other one's is multiplied by zeros, with a scale that is a number
    const i32x8 hi0 = {(int)q.hi[0], (int)q.hi[1], (int)q.hi[2], (int)q.hi[3], 0, 0, 0, 0}, lo0 = {(int)q.lo[0], (int)q.lo[1], (int)q.lo[2], (int)q.lo[3], 0, 0, 0, 0};
    const i32x8 hi1 = {0, 0, 0, 0, (int)q.hi[0], (int)q.hi[1], (int)q.hi[2], (int)q.hi[3]}, lo1 = {0, 0, 0, 0, (int)q.lo[0], (int)q.lo[1], (int)q.lo[2], (int)q.lo[3]};
    const int ks0 = q4 < 2 ? (int)c.ks : 0, ks1 = q4 < 2 ? 0 : (int)c.ks;
    S[0] = q4_score<0>(c.k[0], ks0, hi0, lo0, q.s_hi, q.s_lo, zero);
    S[1] = q4_score<1>(c.k[0], ks1, hi1, lo1, q.s_hi, q.s_lo, zero);
    S[2] = q4_score<2>(c.k[1], ks0, hi0, lo0, q.s_hi, q.s_lo, zero);
    S[3] = q4_score<3>(c.k[1], ks1, hi1, lo1, q.s_hi, q.s_lo, zero);
  }
  // ---- S[T][r] is token 16 q4 + 4 r + T of this lane's head ----
  if (n_tok < CH) {                        // uniform: the sequence's last chunk
    const int left = n_tok - 16 * q4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int T = 0; T < 4; ++T) S[T][r] = 4 * r + T < left ? S[T][r] : -INFINITY;
      // scales of tokens that are not there: whatever the cache holds, no NaN must meet the zeros of P
      const int n = left - 4 * r;
      c.vs[r] = n >= 4 ? c.vs[r] : (n <= 0 ? 0u : c.vs[r] & ((1u << (8 * n)) - 1u));
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int T = 0; T < 4; ++T)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, S[T][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float m_new = fmaxf(m_run, mx * c2);
  // (-inf only where every score so far is: as an underflow or without a number)
  const float ref = m_new == -INFINITY ? 0.f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(m_run - ref);
  m_run = m_new;
  float rowsum = 0.f;
#pragma unroll
  for (int T = 0; T < 4; ++T)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      S[T][r] = __builtin_amdgcn_exp2f(fmaf(S[T][r], c2, -ref));
      rowsum += S[T][r];
    }
  l_run = l_run * alpha + rowsum;
#pragma unroll
  for (int x = 0; x < (GM == 16 ? 2 : 1); ++x)
#pragma unroll
    for (int t = 0; t < D / 32; ++t) O[x][t] *= alpha;

  // ---- O^T += V^T P^T, 16 tokens at a time: k index 8 q4 + 2 r + parity is token 16 q4 + 4 r + T; row i of tile t is the pair of
  // components (head_dim / 16) i + 2 t, + 1 ----
  const q4_column<GM> col(g);
  constexpr uint32_t EVEN = 0x0c0c0302u, ODD = 0x03020c0cu;      // a number's upper half in the lower half of a word, or the upper
  const uint32_t mine = col.odd ? ODD : EVEN;
  const float less = col.rest ? -1.f : 0.f;
  auto tokens = [&](auto tile) {
    constexpr int T = decltype(tile)::value;
    u32x4 P[GM == 4 ? 1 : GM == 8 ? 2 : 4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float x = S[T][r];
      const float top = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
      if constexpr (GM == 4) {
        const uint32_t y = __builtin_bit_cast(uint32_t, fmaf(top, less, x));
        P[0][r] = __builtin_amdgcn_perm(y, y, mine);
      } else {
        const uint32_t y = __builtin_bit_cast(uint32_t, x), z = __builtin_bit_cast(uint32_t, x - top);
        if constexpr (GM == 8) { P[0][r] = __builtin_amdgcn_perm(y, y, mine); P[1][r] = __builtin_amdgcn_perm(z, z, mine); }
        else {
          P[0][r] = y >> 16; P[1][r] = z >> 16;
          P[2][r] = y & 0xffff0000u; P[3][r] = z & 0xffff0000u;
        }
      }
    }
    float sc[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) sc[r] = q4_scale_byte<T>(c.vs[r]);
    auto pair = [&](auto sel) {
      constexpr int t = decltype(sel)::value;
      u32x4 a;
#pragma unroll
      for (int r = 0; r < 4; ++r) a[r] = q4_expand<t>(c.v[4 * r + T], sc[r]);
      const bf16x8 vf = __builtin_bit_cast(bf16x8, a);
      constexpr int NB = GM == 4 ? 1 : 2;
#pragma unroll
      for (int x = 0; x < (GM == 16 ? 2 : 1); ++x)
#pragma unroll
        for (int i = 0; i < NB; ++i) O[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, P[NB * x + i]), O[x][t], 0, 0, 0);
    };
    pair(std::integral_constant<int, 0>{});
    pair(std::integral_constant<int, 1>{});
    if constexpr (D == 128) {
      pair(std::integral_constant<int, 2>{});
      pair(std::integral_constant<int, 3>{});
    }
  };
  tokens(std::integral_constant<int, 0>{});
  tokens(std::integral_constant<int, 1>{});
  tokens(std::integral_constant<int, 2>{});
  tokens(std::integral_constant<int, 3>{});
}

// Partial outputs in LDS: rows of dec_o_at, inside which a row's 32 components stand in the order in which lanes have them:
// parity, row of the tile, tile.
template <int D>
__device__ __forceinline__ int q4_o_at(int wave, int G, int gg, int d) {
  const int in = d & 31;
  const int pos = D == 128 ? (in & 1) * 16 + (in >> 3) * 4 + (in >> 1 & 3) : (in & 16) + (in & 1) * 8 + (in >> 2 & 3) * 2 + (in >> 1 & 1);
  return dec_o_at<D>(wave, G, gg, d - in) + pos;
}
template <int D>
__device__ __forceinline__ void q4_stash(float* s_o, int wave, int G, int head, bool odd, int q4, const f32x4 (&O)[D / 32]) {
  if constexpr (D == 128) {
    f32x4* to = reinterpret_cast<f32x4*>(s_o + dec_o_at<D>(wave, G, head, 32 * q4) + (odd ? 16 : 0));
#pragma unroll
    for (int r = 0; r < 4; ++r) to[r] = f32x4{O[0][r], O[1][r], O[2][r], O[3][r]};
  } else {
    f32x4* to = reinterpret_cast<f32x4*>(s_o + dec_o_at<D>(wave, G, head, 32 * (q4 >> 1)) + (q4 & 1) * 16 + (odd ? 8 : 0));
#pragma unroll
    for (int r = 0; r < 4; r += 2) to[r / 2] = f32x4{O[0][r], O[1][r], O[0][r + 1], O[1][r + 1]};
  }
}

// D: head_dim; GM: query heads that fit the columns; NWV: wavefronts of a workgroup
template <int D, int GM, int NWV>
__global__ __launch_bounds__(64 * NWV, GM == 16 ? 2 : 4) void pa_decode_q4_kernel(q4_params p) {
  __shared__ float s_m[NWV][MAXG], s_l[NWV][MAXG];
  extern __shared__ __attribute__((aligned(16))) float s_o[];    // [NWV][G][D/32][OROW]
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane & 15, q4 = lane >> 4;
  const int G = p.d.G;
  const q4_column<GM> col(g);

  const int len = p.d.kv_len[b];
  u32x4 qx[D / 32];
  const dec_buf qb = dec_buffer(p.d.q + ((int64_t)b * p.d.hq + (int64_t)kvh * G) * D, G * 2 * D);    // (no such head: zeros)
#pragma unroll
  for (int i = 0; i < D / 32; ++i) qx[i] = dec_load16(qb, col.head * 2 * D + 32 * q4, 16 * (i & 1) + 128 * (i >> 1));
  const dec_row row = dec_row_of(p.d, len);
  const int n_slots = len > 0 ? row.n_slots : 0;                 // an empty sequence attends nothing

  float m_run = -INFINITY, l_run = 0.f;
  f32x4 O[GM == 16 ? 2 : 1][D / 32];
#pragma unroll
  for (int x = 0; x < (GM == 16 ? 2 : 1); ++x)
#pragma unroll
    for (int t = 0; t < D / 32; ++t) O[x][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // chunk `slot` of the row requested; the tokens of it that are attended (0: there is no such chunk)
  q4_chunk<D> c;
  auto request = [&](int slot) -> int {
    if (slot >= n_slots) return 0;
    const dec_place pl = dec_place_of(p.d, row, slot);
    if (pl.n_tok <= 0) return 0;                                 // in the diagonal block beyond the query: the row's last ones
    q4_issue<D>(c, p, dec_page(p.d, b, pl.blk), kvh, pl.sub, pl.n_tok, g, q4);
    return pl.n_tok;
  };
  // (The next chunk requested before this one is used, in registers of its own: no gain, 40 to 100 registers more.)
  int slot = wave * p.d.splits + split;
  int n_tok = request(slot);
  const q4_query<D> q = q4_split_query<D>(qx);                   // (while the chunk is on its way)
  while (n_tok > 0) {
    q4_consume<D, GM>(c, q, n_tok, p.d.c2, g, q4, m_run, l_run, O);
    n_tok = request(slot += NWV * p.d.splits);
  }

  // ---- the wavefronts' partials meet in LDS ----
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if (GM == 4) {                                                 // the two parts of P
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) O[0][t][r] += __shfl_xor(O[0][t][r], 8);
  }
  if (col.head < G && !col.rest) {
    if (q4 == 0 && !col.odd) { s_m[wave][col.head] = m_run; s_l[wave][col.head] = l_run; }
    q4_stash<D>(s_o, wave, G, col.head, col.odd, q4, O[0]);
    if constexpr (GM == 16) q4_stash<D>(s_o, wave, G, col.head, true, q4, O[1]);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * D; e += 64 * NWV) {
    const int gg = e / D, d = e % D;
    float M = -INFINITY, L = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < NWV; ++w) M = fmaxf(M, s_m[w][gg]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < NWV; ++w) {
      const float wt = __builtin_amdgcn_exp2f(s_m[w][gg] - ref);
      L = fmaf(wt, s_l[w][gg], L);
      acc = fmaf(wt, s_o[q4_o_at<D>(w, G, gg, d)], acc);
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

// Adds up the splits' partials: one wavefront per (sequence, query head).  The maxima and sums of 64 splits are read by the 64
// lanes at once, the partial outputs eight at a time.
template <int D>
__global__ __launch_bounds__(64) void pa_decode_q4_merge_kernel(dec_params p) {
  constexpr int DPL = D / 64;
  const int64_t h = (int64_t)blockIdx.y * p.hq + blockIdx.x;
  const int lane = threadIdx.x;
  const float* part = p.partials + h * p.splits * (D + 2);
  float M = -INFINITY, L = 0.f, acc[DPL] = {};
  for (int s0 = 0; s0 < p.splits; s0 += 64) {
    const int n = min(64, p.splits - s0);
    const float* ps = part + (int64_t)s0 * (D + 2);
    float m = -INFINITY, l = 0.f;
    if (lane < n) { m = ps[lane * (D + 2) + D]; l = ps[lane * (D + 2) + D + 1]; }
    float top = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float M_new = fmaxf(M, top), ref = M_new == -INFINITY ? 0.f : M_new;
    const float alpha = __builtin_amdgcn_exp2f(M - ref), wt = __builtin_amdgcn_exp2f(m - ref);
    M = M_new;
    float sum = wt * l;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    L = L * alpha + sum;
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] *= alpha;
    for (int s = 0; s < n; s += 8) {
      float o[8][DPL];
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int e = 0; e < DPL; ++e) o[x][e] = s + x < n ? ps[(s + x) * (D + 2) + lane + 64 * e] : 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float w = __shfl(wt, s + x);                 // (a split that is not there: 0)
#pragma unroll
        for (int e = 0; e < DPL; ++e) acc[e] = fmaf(w, o[x][e], acc[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) p.o[h * D + lane + 64 * e] = (__bf16)(L == 0.f ? 0.f : acc[e] / L);
  if (p.lse && lane == 0) p.lse[h] = (M + log2f(L)) * 0.69314718055994530942f;
}

// Workgroups of a (sequence, KV head).  One takes about 1.4 us for each round of its eight wavefronts' chunks, and a second kernel
// to add up the partials costs 2.5 to 3: a row is cut into parts of one round, as far as there are compute units for them, where
// that saves three rounds.  us, rows of 24 / 40 / 64 / 128 / 256 / 1000 chunks, 8 pairs, one workgroup 9.9 / 12.9 / 17.1 / 28.0 / 49.6 / 182,
// four 9.5 / 10.2 / 11.3 / 14.3 / 20.2 / 52.7, by this rule 9.9 / 9.8 / 10.2 / 11.0 / 11.9 / 20.0; 128 pairs, one 10.5 / 14.6 /
// 19.6 / 32.1 / 62.3 / 271, two 11.0 / 14.5 / 18.8 / 29.4 / 51.7 / 230, four 13.3 / 16.4 / 20.3 / 30.2 / 52.4 / 235.
int32_t q4_splits(const powattn_pattern* pattern, int32_t batch, int32_t hkv, int64_t capacity) {
  const int32_t mk = powattn_max_k(pattern, capacity);
  if (mk < 1) return 0;
  const int64_t chunks = (int64_t)mk * (pattern->block / CH), rounds = (chunks + NW - 1) / NW;
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  const int64_t room = n_cu / ((int64_t)batch * hkv);
  int64_t s = rounds < room ? rounds : room;
  if (s > 256) s = 256;
  if (s < 2 || rounds - (rounds + s - 1) / s < 3) return 1;
  return (int32_t)s;
}

template <int D, int GM, int NWV>
int launch_as(const q4_params& p, int batch, hipStream_t stream) {
  static std::atomic<unsigned long long> attr_done{0};
  constexpr auto lds = [](int G) { return dec_o_bytes<D>(G) / NW * NWV; };
  if (int st = pa_allow_dynamic_lds(reinterpret_cast<const void*>(&pa_decode_q4_kernel<D, GM, NWV>), lds(GM), attr_done)) return st;
  const dim3 grid((uint32_t)p.d.splits, (uint32_t)p.d.hkv, (uint32_t)batch);
  hipLaunchKernelGGL((pa_decode_q4_kernel<D, GM, NWV>), grid, dim3(64 * NWV), lds(p.d.G), stream, p);
  if (int st = pa_note_hip(hipGetLastError())) return st;
  if (p.d.splits == 1) return POWATTN_OK;
  hipLaunchKernelGGL((pa_decode_q4_merge_kernel<D>), dim3((uint32_t)p.d.hq, (uint32_t)batch), dim3(64), 0, stream, p.d);
  return pa_note_hip(hipGetLastError());
}
// Four wavefronts instead of eight where every compute unit has two pairs of four rounds or less: more of them are under way, so
// that one's start and end run under the others' chunks (us, 1024 pairs 20.0 / 21.0, 512 pairs 12.6 / 13.3; 512 pairs of 56 chunks 33.0 /
// 32.3, 256 pairs 10.8 / 9.6; head_dim 64, 512 pairs 9.9 / 9.5).
template <int D, int GM>
int launch_q4(const q4_params& p, int batch, int64_t chunks, hipStream_t stream) {
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  if constexpr (D == 128)
    if (p.d.splits == 1 && chunks <= 2 * NW && (int64_t)batch * p.d.hkv >= 2 * (int64_t)n_cu) return launch_as<D, GM, NW / 2>(p, batch, stream);
  return launch_as<D, GM, NW>(p, batch, stream);
}
template <int D>
int launch_d(const q4_params& p, int batch, int64_t chunks, hipStream_t stream) {
  if (p.d.G <= 4) return launch_q4<D, 4>(p, batch, chunks, stream);
  if (p.d.G <= 8) return launch_q4<D, 8>(p, batch, chunks, stream);
  return launch_q4<D, 16>(p, batch, chunks, stream);
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
  const int64_t chunks = (int64_t)powattn_max_k(pattern, capacity) * d.subs;
  return head_dim == 128 ? launch_d<128>(p, batch, chunks, stream) : launch_d<64>(p, batch, chunks, stream);
}
