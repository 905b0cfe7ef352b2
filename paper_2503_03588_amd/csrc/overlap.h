// Whether tensors share memory, for the calls that refuse outputs in the place of inputs or of one another (host code only).
#pragma once
#include <stdint.h>
#include <algorithm>

// a and na bytes from it on, b and nb bytes
inline bool pa_ranges_meet(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x <= y ? y - x < (uintptr_t)na : x - y < (uintptr_t)nb;
}

// Rows of head_dim components [batch, heads, rows] with any strides (in elements).
struct pa_rows { const void* p; int64_t sb, sh, sr; int32_t heads; };

// Whether a row of `a` shares a byte with a row of `b`: whether their distance, delta + the steps along b's dimensions - those along
// a's, can be shorter than a row.  A dimension in which both step alike is one of differences.  The longest steps are
// chosen first, and of each only the few that the shorter ones can make up for, so that two views of one projection take
// a handful of trials.  Layouts that interleave so irregularly that `most` trials do not tell count as meeting.
class pa_rows_trial {
  struct dim { int64_t step, lo, hi; } d[6];
  int n = 0;
  int64_t lo[7], hi[7], row;             // what dimensions i, i + 1 .. can add at least and at most; a row's bytes
  int left;
  void add(int64_t step, int64_t from, int64_t to) {
    if (step < 0) { step = -step; std::swap(from, to); from = -from; to = -to; }
    if (step != 0 && from < to) d[n++] = {step, from, to};
  }
  static int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }
  bool from(int i, int64_t at) {
    if (at + hi[i] <= -row || at + lo[i] >= row) return false;
    if (i == n || left-- <= 0) return true;
    const int64_t s = d[i].step;
    const int64_t k0 = std::max(d[i].lo, -floor_div(at + hi[i + 1] + row - 1, s)), k1 = std::min(d[i].hi, floor_div(row - 1 - at - lo[i + 1], s));
    for (int64_t k = k0; k <= k1; ++k)
      if (from(i + 1, at + k * s)) return true;
    return false;
  }

 public:
  bool meet(const pa_rows& a, const pa_rows& b, int64_t batch, int64_t rows, int32_t head_dim, int32_t elem, int most) {
    const int64_t sa[3] = {a.sb, a.sh, a.sr}, sb[3] = {b.sb, b.sh, b.sr}, na[3] = {batch, a.heads, rows}, nb[3] = {batch, b.heads, rows};
    const int64_t delta = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    row = (int64_t)head_dim * elem;
    int64_t least = delta, farthest = delta;               // memory that is apart altogether: most calls
    for (int i = 0; i < 3; ++i) {
      const int64_t x = (1 - na[i]) * sa[i] * elem, y = (nb[i] - 1) * sb[i] * elem;
      least += std::min<int64_t>(x, 0) + std::min<int64_t>(y, 0);
      farthest += std::max<int64_t>(x, 0) + std::max<int64_t>(y, 0);
    }
    if (least >= row || farthest <= -row) return false;
    for (int i = 0; i < 3; ++i) {
      if (sa[i] == sb[i]) add(sa[i] * elem, 1 - na[i], nb[i] - 1);
      else { add(sa[i] * elem, 1 - na[i], 0); add(sb[i] * elem, 0, nb[i] - 1); }
    }
    std::sort(d, d + n, [](const dim& x, const dim& y) { return x.step > y.step; });
    lo[n] = hi[n] = 0;
    for (int i = n - 1; i >= 0; --i) { lo[i] = lo[i + 1] + d[i].step * d[i].lo; hi[i] = hi[i + 1] + d[i].step * d[i].hi; }
    left = most;
    return from(0, delta);
  }
};
inline bool pa_rows_meet(const pa_rows& a, const pa_rows& b, int64_t batch, int64_t rows, int32_t head_dim, int32_t elem, int most = 1 << 14) {
  return pa_rows_trial().meet(a, b, batch, rows, head_dim, elem, most);
}
