// Split-K decode over a paged cache held in 4 bits (format: q4.h): the step of decode.hip with pages of 4-bit keys and values.
//
// A step reads 2 * (head_dim / 2 + head_dim / 32) bytes per attended token and KV head, 0.27 of the bf16 step's, so that
// it is bound by latency and by the instructions of expanding the cache (about 430 a chunk) rather than by memory,
// until there are enough sequences.  Keys and values are expanded to bf16 in registers, exactly (a 4-bit value
// times a power of two is a bf16 number), and multiplied with v_mfma_f32_16x16x32_bf16.  us, blocks of 64, from a graph, one
// sequence of 32001 tokens / 16 of 65536 / 128 of 1000 .. 16384: 32 query heads on 8 6.5 / 7.8 / 20.7 (4.3 TB/s), 28 on 4 (GM = 8) 6.9 /
// 8.0 / 13.4, 64 on 4 (GM = 16) - / - / 18.5; 32 on 8, blocks of 256, 64 of 10000 .. 30000: 34 (4.8 TB/s).
//  * A chunk is 64 tokens of a block; a wavefront requests all of one before it uses any.  Token 4i + T of it is row i of tile T
//    (T = 0..3) of S^T = K q^T: a lane's piece of a K row lies in one scale's 32 components, the scales of its four tiles are
//    the bytes of one word, and lane (g, q4) (g = lane % 16, q4 = lane / 16) then has the scores of tokens 16 q4 .. 16 q4 + 15.
//    (The scaled 4-bit product, with the query as the sum of two 8-bit rows, needs no conversions, but it does not
//    keep 32 bits of its sums: scores were off by up to 2^-13 of the sum of magnitudes where the query's components differ in size.)
//  * The conversion yields two neighbouring components of a token.  For V the product wants pairs along the tokens: a token
//    counts twice in its sum, once for each component, and P is held with zeros in the other place: O_even and O_odd are
//    different columns.  (Bringing pairs of tokens together by byte permutes: 64 more instructions a chunk, as many products.)
//  * P is multiplied in two parts, its nearest bf16 number and the nearest to what is left: off by at most 2^-17 of it, to either
//    side, instead of bf16's 2^-8 (which would add as much again to the error of the bf16 output).  (Both parts cut, not rounded: one sequence
//    6.43 us instead of 6.50, but up to 2^-15 off, always towards zero, while l_run sums P as it is.)  Up to 4 query heads (GM = 4): 16
//    columns are 4 heads x even, odd x the two parts; up to 8 (GM = 8): two products; up to 16: four.
//  * The wavefronts' partial (max, sum, O) meet in LDS.
#include <math.h>
#include <type_traits>
#include "decode.h"
#include "q4.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct q4_params {
  dec_params d;                          // (k, v, packets, gen are not used)
  const uint8_t* k; const uint8_t* v; const uint8_t* ks; const uint8_t* vs;
};

// A chunk's registers.  Rows behind the last attended token are not read (a buffer load answers zeros).
//   k   head_dim / 4 components ((head_dim / 4) q4 ..) of token 4g + T;  ks  the scales of tokens 4g .. 4g + 3 for them
//   v   head_dim / 16 components of tokens 16 q4 + j;  vs  their 16 scales
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
  c.ks = __builtin_amdgcn_raw_buffer_load_b32(ksb, (D == 128 ? q4 : q4 >> 1) * p.d.B + 4 * g, 0, 0);
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    if constexpr (D == 128) c.k[T] = dec_load16(kb, 4 * g * ROW + 16 * q4, T * ROW);
    else c.k[T] = __builtin_amdgcn_raw_buffer_load_b64(kb, 4 * g * ROW + 8 * q4 + T * ROW, 0, 0);
  }
  c.vs = dec_load16(vsb, (D == 128 ? g >> 2 : g >> 3) * p.d.B + 16 * q4, 0);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if constexpr (D == 128) c.v[j] = __builtin_amdgcn_raw_buffer_load_b32(vb, 16 * q4 * ROW + 4 * g + j * ROW, 0, 0);
    else c.v[j] = __builtin_amdgcn_raw_buffer_load_b16(vb, 16 * q4 * ROW + 2 * g + j * ROW, 0, 0);
  }
  __builtin_amdgcn_sched_barrier(0);       // every load is under way before the first product
}

// byte BYTE of a word of scales as the conversions want it: they look at the exponent's bits only, so what else is shifted
// along does not matter (checked for every code)
template <int BYTE>
__device__ __forceinline__ float q4_scale_byte(uint32_t word) {
  return __builtin_bit_cast(float, BYTE == 3 ? word >> 1 : word << (23 - 8 * BYTE));
}

// two numbers rounded to bf16 (to the nearest, ties to even)
__device__ __forceinline__ uint32_t q4_two(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, q4_bf16x2));
}

// A tile of scores: step s of the product is components (head_dim / 4) q4 + 8 s ..
template <int D, int T>
__device__ __forceinline__ f32x4 q4_score(const q4_chunk<D>& c, const bf16x8 (&qf)[D / 32]) {
  const float sc = q4_scale_byte<T>(c.ks);
  f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const uint32_t w = c.k[T][s];
    const u32x4 a = {q4_expand<0>(w, sc), q4_expand<1>(w, sc), q4_expand<2>(w, sc), q4_expand<3>(w, sc)};
    S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), qf[s], S, 0, 0, 0);
  }
  return S;
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
__device__ __forceinline__ void q4_consume(q4_chunk<D>& c, const bf16x8 (&qf)[D / 32], int n_tok, float c2, int g, int q4,
                                           float& m_run, float& l_run, f32x4 (&O)[GM == 16 ? 2 : 1][D / 32]) {
  f32x4 S[4] = {q4_score<D, 0>(c, qf), q4_score<D, 1>(c, qf), q4_score<D, 2>(c, qf), q4_score<D, 3>(c, qf)};
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
  // of a pair of numbers, the first in the lower half of a word (even) or in the upper (odd), and the second
  const uint32_t first = col.odd ? 0x01000c0cu : 0x0c0c0100u, second = col.odd ? 0x03020c0cu : 0x0c0c0302u;
  const float less = col.rest ? -1.f : 0.f;
  auto tokens = [&](auto tile) {
    constexpr int T = decltype(tile)::value;
    u32x4 P[GM == 4 ? 1 : GM == 8 ? 2 : 4];
#pragma unroll
    for (int r = 0; r < 4; r += 2) {
      const float x0 = S[T][r], x1 = S[T][r + 1];
      const uint32_t top = q4_two(x0, x1);
      const float top0 = __builtin_bit_cast(float, top << 16), top1 = __builtin_bit_cast(float, top & 0xffff0000u);
      if constexpr (GM == 4) {
        const uint32_t y = q4_two(fmaf(top0, less, x0), fmaf(top1, less, x1));
        P[0][r] = __builtin_amdgcn_perm(y, y, first);
        P[0][r + 1] = __builtin_amdgcn_perm(y, y, second);
      } else {
        const uint32_t rest = q4_two(x0 - top0, x1 - top1);
        if constexpr (GM == 8) {
          P[0][r] = __builtin_amdgcn_perm(top, top, first); P[0][r + 1] = __builtin_amdgcn_perm(top, top, second);
          P[1][r] = __builtin_amdgcn_perm(rest, rest, first); P[1][r + 1] = __builtin_amdgcn_perm(rest, rest, second);
        } else {
          P[0][r] = top & 0xffffu; P[0][r + 1] = top >> 16;
          P[1][r] = rest & 0xffffu; P[1][r + 1] = rest >> 16;
          P[2][r] = top << 16; P[2][r + 1] = top & 0xffff0000u;
          P[3][r] = rest << 16; P[3][r + 1] = rest & 0xffff0000u;
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

// D: head_dim; GM: query heads that fit the columns.  (Four or sixteen wavefronts instead of eight: one sequence 7.4 or 8.1 us
// instead of 6.4; 1024 pairs level with four.)
template <int D, int GM>
__global__ __launch_bounds__(64 * NW, GM == 16 ? 2 : 4) void pa_decode_q4_kernel(q4_params p) {
  __shared__ float s_m[NW][MAXG], s_l[NW][MAXG];
  extern __shared__ __attribute__((aligned(16))) float s_o[];    // [NW][G][D/32][OROW]
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane & 15, q4 = lane >> 4;
  const int G = p.d.G;
  const q4_column<GM> col(g);

  const int len = p.d.kv_len[b];
  bf16x8 qf[D / 32];
  const dec_buf qb = dec_buffer(p.d.q + ((int64_t)b * p.d.hq + (int64_t)kvh * G) * D, G * 2 * D);    // (no such head: zeros)
#pragma unroll
  for (int s = 0; s < D / 32; ++s) qf[s] = __builtin_bit_cast(bf16x8, dec_load16(qb, col.head * 2 * D + (D / 2) * q4, 16 * s));
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
  while (n_tok > 0) {
    q4_consume<D, GM>(c, qf, n_tok, p.d.c2, g, q4, m_run, l_run, O);
    n_tok = request(slot += NW * p.d.splits);
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

// Workgroups of a (sequence, KV head).  One takes about 1.7 us for each round of its eight wavefronts' chunks, and a second kernel
// to add up the partials costs 2 to 3: a row is cut into parts of one round, as far as there are compute units for them, where
// that saves two rounds.  us, rows of 24 / 40 / 64 / 128 / 256 / 1000 chunks, 8 pairs, one workgroup 9.9 / 13.3 / 19.0 / 33.2 / 61.3 / 234,
// four 8.9 / 9.6 / 11.2 / 15.0 / 22.2 / 67.6, parts of one round 9.1 / 9.3 / 9.6 / 10.3 / 11.3 / 20.3; 128 pairs, one 10.4 / 15.0 / 21.5 /
// 37.0 / 75.8 / 308, two 10.5 / 14.8 / 19.3 / 29.7 / 52.6 / 233, four 12.2 / 16.2 / 20.0 / 30.8 / 55.5 / 237; 13 chunks, 8 pairs, one 6.4, two 8.3.
int32_t q4_splits(const powattn_pattern* pattern, int32_t batch, int32_t hkv, int64_t capacity) {
  const int32_t mk = powattn_max_k(pattern, capacity);
  if (mk < 1) return 0;
  const int64_t chunks = (int64_t)mk * (pattern->block / CH), rounds = (chunks + NW - 1) / NW;
  int n_cu = 1;
  pa_current_device(nullptr, &n_cu);
  const int64_t room = n_cu / ((int64_t)batch * hkv);
  int64_t s = rounds < room ? rounds : room;
  if (s > 256) s = 256;
  if (s < 2 || rounds - (rounds + s - 1) / s < 2) return 1;
  return (int32_t)s;
}

template <int D, int GM>
int launch_q4(const q4_params& p, int batch, hipStream_t stream) {
  static std::atomic<unsigned long long> attr_done{0};
  if (int st = pa_allow_dynamic_lds(reinterpret_cast<const void*>(&pa_decode_q4_kernel<D, GM>), dec_o_bytes<D>(GM), attr_done)) return st;
  const dim3 grid((uint32_t)p.d.splits, (uint32_t)p.d.hkv, (uint32_t)batch);
  hipLaunchKernelGGL((pa_decode_q4_kernel<D, GM>), grid, dim3(64 * NW), dec_o_bytes<D>(p.d.G), stream, p);
  if (int st = pa_note_hip(hipGetLastError())) return st;
  if (p.d.splits == 1) return POWATTN_OK;
  hipLaunchKernelGGL((pa_decode_q4_merge_kernel<D>), dim3((uint32_t)p.d.hq, (uint32_t)batch), dim3(64), 0, stream, p.d);
  return pa_note_hip(hipGetLastError());
}
template <int D>
int launch_d(const q4_params& p, int batch, hipStream_t stream) {
  return p.d.G <= 4 ? launch_q4<D, 4>(p, batch, stream) : p.d.G <= 8 ? launch_q4<D, 8>(p, batch, stream) : launch_q4<D, 16>(p, batch, stream);
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
  return head_dim == 128 ? launch_d<128>(p, batch, stream) : launch_d<64>(p, batch, stream);
}
