// Norm of every query and key head and the rotation by its position, in one pass, and the gradients.
//   n = x r, r = 1 / sqrt(mean(x^2) + eps);  u = w n;  y = the rotation of u's first rot_dim components by position * inv_freq
//   du = the rotation back of dy;  dw = sum over all rows of du n;  dn = w du;  dx = r (dn - n mean(dn n))
// with pairs (i, i + rot_dim / 2), or (2i, 2i + 1) where POWATTN_ROPE_INTERLEAVED is set.
//
// Bound by memory: 2 (gradients: 3) passes over the tensors (32768 rows of 32 heads of 128 in bf16: 102 us, 5.2 TB/s; gradients 171,
// 4.7).  A row of head_dim components belongs to 8 (head_dim 64: 4)
// lanes, 16 components each in two pieces of 8, chosen so that both halves of a pair are in one lane; a wavefront has 8
// (16) consecutive tokens of a head, and walks through the heads with the same angles.  An angle is the exact product of
// the position and the frequency, reduced to a part of a turn in 64 bits (in 32 bits a position of a million is known to a
// sixteenth of a radian); everything else is in 32 bits, rounded once at the end.
#include <math.h>
#include "common.h"
#include "overlap.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int THREADS = 256;
constexpr int AHEAD = 2;                 // heads whose rows are requested together, while those before them are in use

// rows [batch, heads, rows, head_dim], strides in elements
struct nr_rows { const void* p; int64_t sb, sh, sr; };
struct nr_out { void* p; int64_t sb, sh, sr; };
struct nr_params {
  nr_rows x[2];                          // queries, keys
  const void* w[2];
  nr_rows dy[2];                         // gradients only
  nr_out out[2];                         // y, or dx
  const float* inv_freq; const int32_t* q_start; const int32_t* q_len;
  float* partials[2];                    // gradients: [parts of this kind, head_dim] sums of dw
  int32_t heads[2], chunks[2], per_chunk[2];   // heads, their chunks (a workgroup's), heads of a chunk
  int32_t n_tokens, rows, rot;
  float eps;
};

// ---- 8 components ----
template <class T> struct raw8;
template <> struct raw8<__bf16> { u32x4 a; };
template <> struct raw8<float> { u32x4 a, b; };

template <bool VEC>
__device__ __forceinline__ void nr_load(raw8<__bf16>& r, const __bf16* p) {
  if constexpr (VEC) r.a = *reinterpret_cast<const u32x4*>(p);
  else {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.a[i] = (uint32_t)q[2 * i] | (uint32_t)q[2 * i + 1] << 16;
  }
}
template <bool VEC>
__device__ __forceinline__ void nr_load(raw8<float>& r, const float* p) {
  if constexpr (VEC) {
    r.a = reinterpret_cast<const u32x4*>(p)[0];
    r.b = reinterpret_cast<const u32x4*>(p)[1];
  } else {
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.a[i] = q[i]; r.b[i] = q[4 + i]; }
  }
}
__device__ __forceinline__ void nr_floats(float (&f)[8], const raw8<__bf16>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __builtin_bit_cast(float, r.a[i] << 16);
    f[2 * i + 1] = __builtin_bit_cast(float, r.a[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void nr_floats(float (&f)[8], const raw8<float>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = r.a[i], b = r.b[i];         // (a bit cast of a vector's element reads its first one)
    f[i] = __builtin_bit_cast(float, a);
    f[4 + i] = __builtin_bit_cast(float, b);
  }
}
// MODE 0: components one at a time, 1: 16 bytes at a time, 2: the same past the caches
template <int MODE>
__device__ __forceinline__ void nr_put16(void* p, u32x4 x) {
  if constexpr (MODE == 2) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = x;
}
template <int MODE>
__device__ __forceinline__ void nr_store(__bf16* p, const float (&f)[8]) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  bf16x8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (__bf16)f[i];
  if constexpr (MODE > 0) nr_put16<MODE>(p, __builtin_bit_cast(u32x4, y));
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = y[i];
  }
}
template <int MODE>
__device__ __forceinline__ void nr_store(float* p, const float (&f)[8]) {
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  if constexpr (MODE > 0) {
    nr_put16<MODE>(p, __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]}));
    nr_put16<MODE>(p + 4, __builtin_bit_cast(u32x4, f32x4{f[4], f[5], f[6], f[7]}));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = f[i];
  }
}

// Where lane c of a row has its two pieces, and whether they are rotated (rot_dim is a multiple of 16: all of them or none).
// Pairs: lane c has pairs 8c .. 8c + 7; the components behind rot_dim make up the remaining "pairs".
template <bool INTER>
struct nr_place {
  int a, b; bool turned;
  __device__ __forceinline__ nr_place(int c, int rot, int D) {
    turned = 16 * c < rot;
    if (INTER) { a = 16 * c; b = a + 8; }
    else {
      a = turned ? 8 * c : rot / 2 + 8 * c;
      b = (turned ? rot / 2 : D / 2) + 8 * c;
    }
  }
};
// cos and sin of the lane's eight angles at a position
__device__ __forceinline__ void nr_angles(float (&cs)[8], float (&sn)[8], const double (&turns)[8], int64_t pos) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double t = (double)pos * turns[i];
    sincospif(2.f * (float)(t - rint(t)), &sn[i], &cs[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void nr_turns(double (&turns)[8], const float* inv_freq, int c, bool turned) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = 0.f;
  if (turned) {
    raw8<float> r;
    nr_load<VEC>(r, inv_freq + 8 * c);
    nr_floats(f, r);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) turns[i] = (double)f[i] * 0.15915494309189533577;      // 1 / 2 pi
}
template <bool INTER>
__device__ __forceinline__ void nr_rotate(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& x = INTER ? (i < 4 ? a[2 * i] : b[2 * i - 8]) : a[i];
    float& y = INTER ? (i < 4 ? a[2 * i + 1] : b[2 * i - 7]) : b[i];
    const float u = x, v = y;
    x = u * cs[i] - v * sn[i];
    y = u * sn[i] + v * cs[i];
  }
}
template <int LANES>
__device__ __forceinline__ float nr_sum(float x) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

template <class T, int D, int MODE, bool INTER>
__global__ __launch_bounds__(THREADS) void pa_qk_norm_rope_kernel(nr_params p) {
  constexpr int LPR = D / 16;
  constexpr bool VEC = MODE > 0;
  const int c = threadIdx.x % LPR;
  const int t = blockIdx.x * (THREADS / LPR) + threadIdx.x / LPR;
  int chunk = blockIdx.y;
  const int which = chunk >= p.chunks[0];
  chunk -= which ? p.chunks[0] : 0;
  const int h0 = chunk * p.per_chunk[which], h1 = min(h0 + p.per_chunk[which], p.heads[which]);
  if (t >= p.n_tokens) return;             // (whole rows: the lanes of a row stay together)
  const unsigned b = (unsigned)t / (unsigned)p.rows, r = (unsigned)t - b * (unsigned)p.rows;
  if (p.q_len && (int)r >= p.q_len[b]) return;
  const nr_place<INTER> at(c, p.rot, D);

  raw8<T> wa, wb;
  nr_load<VEC>(wa, (const T*)p.w[which] + at.a);
  nr_load<VEC>(wb, (const T*)p.w[which] + at.b);
  double turns[8];
  float cs[8], sn[8];
  nr_turns<VEC>(turns, p.inv_freq, c, at.turned);
  const T* x = (const T*)p.x[which].p + b * p.x[which].sb + r * p.x[which].sr;
  T* y = (T*)p.out[which].p + b * p.out[which].sb + r * p.out[which].sr;
  const int64_t xh = p.x[which].sh, yh = p.out[which].sh;
  raw8<T> ra[AHEAD], rb[AHEAD], na[AHEAD], nb[AHEAD];
  auto request = [&](raw8<T> (&u)[AHEAD], raw8<T> (&v)[AHEAD], int h) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (h + i >= h1) break;
      nr_load<VEC>(u[i], x + (h + i) * xh + at.a);
      nr_load<VEC>(v[i], x + (h + i) * xh + at.b);
    }
  };
  // (under way while the angles are formed; with a q_start the angles wait for it, and thereby for the rows requested before it)
  request(ra, rb, h0);
  nr_angles(cs, sn, turns, (int64_t)(p.q_start ? p.q_start[b] : 0) + r);
  float w0[8], w1[8];
  nr_floats(w0, wa);
  nr_floats(w1, wb);

  for (int h = h0; h < h1; h += AHEAD) {
    request(na, nb, h + AHEAD);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (h + i >= h1) break;
      float f0[8], f1[8], ss = 0.f;
      nr_floats(f0, ra[i]);
      nr_floats(f1, rb[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(f0[e], f0[e], fmaf(f1[e], f1[e], ss));
      const float rn = 1.f / sqrtf(nr_sum<LPR>(ss) * (1.f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) { f0[e] = f0[e] * rn * w0[e]; f1[e] = f1[e] * rn * w1[e]; }
      if (at.turned) nr_rotate<INTER>(f0, f1, cs, sn);
      nr_store<MODE>(y + (h + i) * yh + at.a, f0);
      nr_store<MODE>(y + (h + i) * yh + at.b, f1);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) { ra[i] = na[i]; rb[i] = nb[i]; }
  }
}

// Gradients: a workgroup walks through every gridDim.x-th group of tokens with its heads, keeps its sums of dw in registers
// and leaves them in the workspace; the sums of all workgroups are added by the kernel below, in a fixed order.  (The next
// head's rows requested ahead, as above, cost a third of the wavefronts: 32768 rows 175 -> 169 us, 1000 13.5 -> 16.9, 8192 61.7 -> 64.3.)
template <class T, int D, int MODE, bool INTER>
__global__ __launch_bounds__(THREADS) void pa_qk_norm_rope_grad_kernel(nr_params p) {
  constexpr int LPR = D / 16, TOK = THREADS / LPR, NWV = THREADS / 64;
  constexpr bool VEC = MODE > 0;
  __shared__ float s_dw[NWV][D];
  const int c = threadIdx.x % LPR;
  int chunk = blockIdx.y;
  const int which = chunk >= p.chunks[0];
  chunk -= which ? p.chunks[0] : 0;
  const int h0 = chunk * p.per_chunk[which], h1 = min(h0 + p.per_chunk[which], p.heads[which]);
  const nr_place<INTER> at(c, p.rot, D);
  raw8<T> wa, wb;
  nr_load<VEC>(wa, (const T*)p.w[which] + at.a);
  nr_load<VEC>(wb, (const T*)p.w[which] + at.b);
  float w0[8], w1[8], dw0[8], dw1[8];
  nr_floats(w0, wa);
  nr_floats(w1, wb);
  double turns[8];
  nr_turns<VEC>(turns, p.inv_freq, c, at.turned);
#pragma unroll
  for (int e = 0; e < 8; ++e) dw0[e] = dw1[e] = 0.f;

  const int64_t xh = p.x[which].sh, gh = p.dy[which].sh, oh = p.out[which].sh;
  for (int64_t t = (int64_t)blockIdx.x * TOK + threadIdx.x / LPR; t < p.n_tokens; t += (int64_t)gridDim.x * TOK) {
    const unsigned b = (unsigned)t / (unsigned)p.rows, r = (unsigned)t - b * (unsigned)p.rows;
    if (p.q_len && (int)r >= p.q_len[b]) continue;
    float cs[8], sn[8];
    nr_angles(cs, sn, turns, (int64_t)(p.q_start ? p.q_start[b] : 0) + r);
#pragma unroll
    for (int e = 0; e < 8; ++e) sn[e] = -sn[e];            // the rotation back
    const T* x = (const T*)p.x[which].p + b * p.x[which].sb + r * p.x[which].sr;
    const T* g = (const T*)p.dy[which].p + b * p.dy[which].sb + r * p.dy[which].sr;
    T* o = (T*)p.out[which].p + b * p.out[which].sb + r * p.out[which].sr;
    for (int h = h0; h < h1; ++h) {
      raw8<T> xa, xb, ga, gb;
      nr_load<VEC>(xa, x + h * xh + at.a);
      nr_load<VEC>(xb, x + h * xh + at.b);
      nr_load<VEC>(ga, g + h * gh + at.a);
      nr_load<VEC>(gb, g + h * gh + at.b);
      float f0[8], f1[8], d0[8], d1[8];
      nr_floats(f0, xa);
      nr_floats(f1, xb);
      nr_floats(d0, ga);
      nr_floats(d1, gb);
      if (at.turned) nr_rotate<INTER>(d0, d1, cs, sn);
      float ss = 0.f, sd = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss = fmaf(f0[e], f0[e], fmaf(f1[e], f1[e], ss));
        sd = fmaf(d0[e] * w0[e], f0[e], fmaf(d1[e] * w1[e], f1[e], sd));
      }
      const float rn = 1.f / sqrtf(nr_sum<LPR>(ss) * (1.f / D) + p.eps);
      const float k = nr_sum<LPR>(sd) * rn * rn * (1.f / D);           // mean(dn n) n = k x
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dw0[e] = fmaf(d0[e], f0[e] * rn, dw0[e]);
        dw1[e] = fmaf(d1[e], f1[e] * rn, dw1[e]);
        d0[e] = rn * (d0[e] * w0[e] - k * f0[e]);
        d1[e] = rn * (d1[e] * w1[e] - k * f1[e]);
      }
      nr_store<MODE>(o + h * oh + at.a, d0);
      nr_store<MODE>(o + h * oh + at.b, d1);
    }
  }

#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int d = LPR; d < 64; d <<= 1) { dw0[e] += __shfl_xor(dw0[e], d); dw1[e] += __shfl_xor(dw1[e], d); }
  }
  const int wave = threadIdx.x / 64;
  if (threadIdx.x % 64 < LPR) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { s_dw[wave][at.a + e] = dw0[e]; s_dw[wave][at.b + e] = dw1[e]; }
  }
  __syncthreads();
  float* part = p.partials[which] + ((int64_t)chunk * gridDim.x + blockIdx.x) * D;
  for (int d = threadIdx.x; d < D; d += THREADS) {
    float s = 0.f;
#pragma unroll
    for (int wv = 0; wv < NWV; ++wv) s += s_dw[wv][d];
    part[d] = s;
  }
}

constexpr int SUM_COLS = 32, SUM_THREADS = 1024;
__global__ __launch_bounds__(SUM_THREADS) void pa_qk_norm_rope_sum_kernel(const float* part_q, const float* part_k, int n_q, int n_k,
                                                                          float* dw_q, float* dw_k, int D) {
  __shared__ float s[SUM_THREADS / SUM_COLS][SUM_COLS];
  const float* part = blockIdx.y ? part_k : part_q;
  const int n = blockIdx.y ? n_k : n_q;
  const int col = threadIdx.x % SUM_COLS, row = threadIdx.x / SUM_COLS, d = blockIdx.x * SUM_COLS + col;
  constexpr int ROWS = SUM_THREADS / SUM_COLS, AT_ONCE = 16;
  float a = 0.f;
  for (int i0 = row; i0 < n; i0 += ROWS * AT_ONCE) {       // a trip to memory for 16 rows
    float x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) x[j] = i0 + j * ROWS < n ? part[(int64_t)(i0 + j * ROWS) * D + d] : 0.f;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) a += x[j];
  }
  s[row][col] = a;
  __syncthreads();
  if (row == 0) {
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) all += s[i][col];
    (blockIdx.y ? dw_k : dw_q)[d] = all;
  }
}

bool aligned(const nr_params& p, bool grad, size_t elem) {
  const int64_t per = 16 / (int64_t)elem;
  bool ok = ((uintptr_t)p.inv_freq & 15u) == 0;
  for (int i = 0; i < 2; ++i) {
    ok = ok && ((uintptr_t)p.w[i] & 15u) == 0;
    ok = ok && ((uintptr_t)p.x[i].p & 15u) == 0 && p.x[i].sb % per == 0 && p.x[i].sh % per == 0 && p.x[i].sr % per == 0;
    ok = ok && ((uintptr_t)p.out[i].p & 15u) == 0 && p.out[i].sb % per == 0 && p.out[i].sh % per == 0 && p.out[i].sr % per == 0;
    if (grad) ok = ok && ((uintptr_t)p.dy[i].p & 15u) == 0 && p.dy[i].sb % per == 0 && p.dy[i].sh % per == 0 && p.dy[i].sr % per == 0;
  }
  return ok;
}

// Heads of a workgroup: as many as leave `want` workgroups in the launch.
void deal_heads(nr_params& p, int64_t token_groups, int64_t want) {
  int64_t chunks = (want + token_groups - 1) / token_groups;         // of all heads together
  const int64_t all = p.heads[0] + p.heads[1];
  if (chunks > all) chunks = all;
  if (chunks < 1) chunks = 1;
  const int32_t per = (int32_t)((all + chunks - 1) / chunks);
  for (int i = 0; i < 2; ++i) {
    p.chunks[i] = (p.heads[i] + per - 1) / per;
    p.per_chunk[i] = (p.heads[i] + p.chunks[i] - 1) / p.chunks[i];
  }
}

struct nr_grid { int64_t groups; uint32_t x; };
// The gradients' launch: the workspace has room for the sums of every workgroup.
nr_grid grad_grid(nr_params& p, int32_t head_dim) {
  const int64_t tok = THREADS / (head_dim / 16);
  nr_grid g;
  g.groups = (p.n_tokens + tok - 1) / tok;
  deal_heads(p, g.groups, 1024);                           // (us, 2048 / 8192 rows of 40 heads, 1024 workgroups 21.6 / 61.2, 640 18.0 / 66.7)
  const int64_t chunks = p.chunks[0] + p.chunks[1];
  int64_t x = (2048 + chunks - 1) / chunks;
  if (x > g.groups) x = g.groups;
  g.x = (uint32_t)x;
  return g;
}

int check_rope(int32_t batch, int32_t hq, int32_t hkv, int64_t rows, int32_t head_dim, int32_t dtype) {
  if (batch < 1 || hq < 1 || hkv < 1 || rows < 1 || head_dim < 1) return POWATTN_INVALID_ARG;
  if (dtype != POWATTN_BF16 && dtype != POWATTN_F32) return POWATTN_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return POWATTN_UNSUPPORTED;
  if (hq > 32767 || hkv > 32767 || rows > 0x7fffffff || (int64_t)batch * rows > 0x7fffffff - 4096) return POWATTN_UNSUPPORTED;
  return POWATTN_OK;
}
int check_rotation(int32_t rot, int32_t head_dim, uint32_t flags, float eps) {
  if (flags & ~POWATTN_ROPE_INTERLEAVED) return POWATTN_INVALID_ARG;
  if (!(eps >= 0.f) || eps > 3.0e38f) return POWATTN_INVALID_ARG;
  if (rot < 0 || rot > head_dim) return POWATTN_INVALID_ARG;
  if (rot % 16 != 0) return POWATTN_UNSUPPORTED;
  return POWATTN_OK;
}

// Whether an output shares memory with one of the tensors that are read, or with the other output.
bool outputs_meet(const nr_params& p, bool grad, int64_t batch, int32_t head_dim, int32_t dtype) {
  const int32_t elem = dtype == POWATTN_F32 ? 4 : 2;
  auto meet = [&](const void* a, const int64_t (&sa)[3], int32_t ha, const void* b, const int64_t (&sb)[3], int32_t hb) {
    return pa_rows_meet({a, sa[0], sa[1], sa[2], ha}, {b, sb[0], sb[1], sb[2], hb}, batch, p.rows, head_dim, elem);
  };
  int64_t so[2][3];
  for (int i = 0; i < 2; ++i) { so[i][0] = p.out[i].sb; so[i][1] = p.out[i].sh; so[i][2] = p.out[i].sr; }
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 2; ++i) {
      const int64_t sx[3] = {p.x[i].sb, p.x[i].sh, p.x[i].sr}, sy[3] = {p.dy[i].sb, p.dy[i].sh, p.dy[i].sr};
      if (meet(p.out[o].p, so[o], p.heads[o], p.x[i].p, sx, p.heads[i])) return true;
      if (grad && meet(p.out[o].p, so[o], p.heads[o], p.dy[i].p, sy, p.heads[i])) return true;
    }
  return meet(p.out[0].p, so[0], p.heads[0], p.out[1].p, so[1], p.heads[1]);
}

template <class T, int D, int MODE>
void launch_forward(const nr_params& p, dim3 grid, bool inter, hipStream_t s) {
  if (inter) hipLaunchKernelGGL((pa_qk_norm_rope_kernel<T, D, MODE, true>), grid, dim3(THREADS), 0, s, p);
  else hipLaunchKernelGGL((pa_qk_norm_rope_kernel<T, D, MODE, false>), grid, dim3(THREADS), 0, s, p);
}
template <class T, int D, int MODE>
void launch_grad(const nr_params& p, dim3 grid, bool inter, hipStream_t s) {
  if (inter) hipLaunchKernelGGL((pa_qk_norm_rope_grad_kernel<T, D, MODE, true>), grid, dim3(THREADS), 0, s, p);
  else hipLaunchKernelGGL((pa_qk_norm_rope_grad_kernel<T, D, MODE, false>), grid, dim3(THREADS), 0, s, p);
}
template <bool GRAD, class T>
void launch_d(const nr_params& p, dim3 grid, int32_t head_dim, int mode, bool inter, hipStream_t s) {
#define GO(D, MODE) do { if constexpr (GRAD) launch_grad<T, D, MODE>(p, grid, inter, s); else launch_forward<T, D, MODE>(p, grid, inter, s); } while (0)
  if (head_dim == 128) { if (mode == 2) GO(128, 2); else if (mode == 1) GO(128, 1); else GO(128, 0); }
  else { if (mode == 2) GO(64, 2); else if (mode == 1) GO(64, 1); else GO(64, 0); }
#undef GO
}
// The outputs go past the caches where the tensors together are larger than half of the 256 MB behind the L2s: what is written
// would push out what is still to be read.  us, through / past, 40 heads of 128 in bf16: 32768 rows (537 MB, 32 heads) 109 / 105, 8192 (168 MB)
// 41.6 / 29.7, their gradients 179 / 175 and 64.4 / 62.1; 8192 rows of 64 (84 MB) 17.0 / 19.9.
template <bool GRAD>
int launch(const nr_params& p, dim3 grid, int32_t head_dim, int32_t dtype, bool inter, hipStream_t s) {
  const int64_t elem = dtype == POWATTN_F32 ? 4 : 2;
  const int64_t bytes = (GRAD ? 3 : 2) * elem * p.n_tokens * head_dim * (p.heads[0] + p.heads[1]);
  const int mode = !aligned(p, GRAD, elem) ? 0 : bytes > (128 << 20) ? 2 : 1;
  if (dtype == POWATTN_F32) launch_d<GRAD, float>(p, grid, head_dim, mode, inter, s);
  else launch_d<GRAD, __bf16>(p, grid, head_dim, mode, inter, s);
  return pa_note_hip(hipGetLastError());
}

}  // namespace

extern "C" int powattn_qk_norm_rope(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides,
                                    const void* q_weight, const void* k_weight, const float* d_inv_freq, int32_t rot_dim,
                                    uint32_t flags, const int32_t* d_q_start, const int32_t* d_q_len, void* q_out, void* k_out,
                                    int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int64_t rows, int32_t head_dim,
                                    int32_t dtype, float eps, void* hip_stream) {
  if (!q || !k || !q_strides || !k_strides || !q_weight || !k_weight || !q_out || !k_out) return POWATTN_INVALID_ARG;
  if (!d_inv_freq && rot_dim != 0) return POWATTN_INVALID_ARG;
  int st = check_rope(batch, n_q_heads, n_kv_heads, rows, head_dim, dtype);
  if (st == POWATTN_OK) st = check_rotation(rot_dim, head_dim, flags, eps);
  if (st != POWATTN_OK) return st;
  nr_params p = {};
  p.x[0] = {q, q_strides[0], q_strides[1], q_strides[2]};
  p.x[1] = {k, k_strides[0], k_strides[1], k_strides[2]};
  p.w[0] = q_weight; p.w[1] = k_weight;
  p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads;
  void* out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) p.out[i] = {out[i], (int64_t)p.heads[i] * rows * head_dim, rows * head_dim, head_dim};
  p.inv_freq = d_inv_freq; p.q_start = d_q_start; p.q_len = d_q_len;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.rot = rot_dim; p.eps = eps;
  if (outputs_meet(p, false, batch, head_dim, dtype)) return POWATTN_INVALID_ARG;
  const int64_t tok = THREADS / (head_dim / 16), groups = (p.n_tokens + tok - 1) / tok;
  deal_heads(p, groups, 1024);
  const dim3 grid((uint32_t)groups, (uint32_t)(p.chunks[0] + p.chunks[1]));
  if ((int64_t)grid.x * grid.y > 0xffffffffLL / THREADS) return POWATTN_UNSUPPORTED;   // a launch has fewer than 2^32 threads
  return launch<false>(p, grid, head_dim, dtype, (flags & POWATTN_ROPE_INTERLEAVED) != 0, (hipStream_t)hip_stream);
}

extern "C" size_t powattn_qk_norm_rope_backward_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int64_t rows,
                                                                int32_t head_dim) {
  if (check_rope(batch, n_q_heads, n_kv_heads, rows, head_dim, POWATTN_BF16) != POWATTN_OK) return 0;
  nr_params p = {};
  p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads; p.n_tokens = (int32_t)(batch * rows);
  const nr_grid g = grad_grid(p, head_dim);
  return (size_t)g.x * (p.chunks[0] + p.chunks[1]) * head_dim * sizeof(float);
}

extern "C" int powattn_qk_norm_rope_backward(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides,
                                             const void* q_weight, const void* k_weight, const float* d_inv_freq, int32_t rot_dim,
                                             uint32_t flags, const int32_t* d_q_start, const int32_t* d_q_len, const void* d_q_out,
                                             const void* d_k_out, void* dq, const int64_t* dq_strides, void* dk,
                                             const int64_t* dk_strides, float* dq_weight, float* dk_weight, int32_t batch,
                                             int32_t n_q_heads, int32_t n_kv_heads, int64_t rows, int32_t head_dim, int32_t dtype,
                                             float eps, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!q || !k || !q_strides || !k_strides || !q_weight || !k_weight || !d_q_out || !d_k_out) return POWATTN_INVALID_ARG;
  if (!dq || !dk || !dq_strides || !dk_strides || !dq_weight || !dk_weight) return POWATTN_INVALID_ARG;
  if (!d_inv_freq && rot_dim != 0) return POWATTN_INVALID_ARG;
  int st = check_rope(batch, n_q_heads, n_kv_heads, rows, head_dim, dtype);
  if (st == POWATTN_OK) st = check_rotation(rot_dim, head_dim, flags, eps);
  if (st != POWATTN_OK) return st;
  const size_t need = powattn_qk_norm_rope_backward_workspace_bytes(batch, n_q_heads, n_kv_heads, rows, head_dim);
  if (!workspace || workspace_bytes < need) return POWATTN_WORKSPACE_TOO_SMALL;
  if (((uintptr_t)workspace & 255u) != 0) return POWATTN_INVALID_ARG;
  nr_params p = {};
  p.x[0] = {q, q_strides[0], q_strides[1], q_strides[2]};
  p.x[1] = {k, k_strides[0], k_strides[1], k_strides[2]};
  p.w[0] = q_weight; p.w[1] = k_weight;
  p.heads[0] = n_q_heads; p.heads[1] = n_kv_heads;
  const void* dy[2] = {d_q_out, d_k_out};
  for (int i = 0; i < 2; ++i) p.dy[i] = {dy[i], (int64_t)p.heads[i] * rows * head_dim, rows * head_dim, head_dim};
  p.out[0] = {dq, dq_strides[0], dq_strides[1], dq_strides[2]};
  p.out[1] = {dk, dk_strides[0], dk_strides[1], dk_strides[2]};
  p.inv_freq = d_inv_freq; p.q_start = d_q_start; p.q_len = d_q_len;
  p.n_tokens = (int32_t)(batch * rows); p.rows = (int32_t)rows; p.rot = rot_dim; p.eps = eps;
  if (outputs_meet(p, true, batch, head_dim, dtype)) return POWATTN_INVALID_ARG;
  const int64_t dw_bytes = head_dim * (int64_t)sizeof(float);
  if (pa_ranges_meet(dq_weight, dw_bytes, dk_weight, dw_bytes)) return POWATTN_INVALID_ARG;
  const nr_grid g = grad_grid(p, head_dim);
  p.partials[0] = (float*)workspace;
  p.partials[1] = p.partials[0] + (int64_t)g.x * p.chunks[0] * head_dim;
  hipStream_t stream = (hipStream_t)hip_stream;
  st = launch<true>(p, dim3(g.x, (uint32_t)(p.chunks[0] + p.chunks[1])), head_dim, dtype, (flags & POWATTN_ROPE_INTERLEAVED) != 0, stream);
  if (st != POWATTN_OK) return st;
  hipLaunchKernelGGL(pa_qk_norm_rope_sum_kernel, dim3((uint32_t)head_dim / SUM_COLS, 2), dim3(SUM_THREADS), 0, stream, p.partials[0], p.partials[1],
                     (int)(g.x * p.chunks[0]), (int)(g.x * p.chunks[1]), dq_weight, dk_weight, head_dim);
  return pa_note_hip(hipGetLastError());
}
