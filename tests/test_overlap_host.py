"""Whether strided rows share memory (csrc/overlap.h, compiled for the CPU), against the bytes written down one by one."""
import itertools
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include "overlap.h"
int main() {
  long long x[14];
  for (;;) {
    for (int i = 0; i < 14; ++i) if (scanf("%lld", x + i) != 1) return 0;
    const pa_rows a = {(void*)x[0], x[1], x[2], x[3], (int)x[4]}, b = {(void*)x[5], x[6], x[7], x[8], (int)x[9]};
    printf("%d\n", (int)pa_rows_meet(a, b, x[10], x[11], (int)x[12], (int)x[13]));
  }
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs a C++ compiler")
    d = tmp_path_factory.mktemp("overlap")
    (d / "overlap.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2503_03588_amd", "csrc"), str(d / "overlap.cpp"), "-o",
                    str(d / "overlap")], check=True, timeout=120)

    def f(cases):
        text = "\n".join(" ".join(map(str, (*a, *b, batch, rows, dim, elem))) for a, b, batch, rows, dim, elem in cases)
        out = subprocess.run([str(d / "overlap")], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [line == "1" for line in out.split()]
    return f


def one_by_one(a, b, batch, rows, dim, elem):
    def held(t):
        p, sb, sh, sr, heads = t
        return {p + (i * sb + h * sh + r * sr) * elem + c for i in range(batch) for h in range(heads) for r in range(rows)
                for c in range(dim * elem)}
    return bool(held(a) & held(b))


def test_small_layouts(meet):
    rng = random.Random(1)
    cases = []
    for _ in range(3000):
        batch, rows, dim, elem = rng.randint(1, 3), rng.randint(1, 4), rng.choice((2, 4)), rng.choice((2, 4))
        heads = rng.randint(1, 3), rng.randint(1, 3)
        strides = [[rng.choice((0, dim, dim + 1, 2 * dim, 3 * dim, 4 * dim, 7 * dim, 13 * dim, 30 * dim, -dim)) for _ in range(3)] for _ in range(2)]
        if rng.random() < 0.5:                             # alike, as views of one tensor are
            strides[1] = list(strides[0])
        at = 4096, 4096 + rng.randint(-40, 40) * (elem if rng.random() < 0.8 else 1)
        cases.append(((at[0], *strides[0], heads[0]), (at[1], *strides[1], heads[1]), batch, rows, dim, elem))
    want = [one_by_one(*c) for c in cases]
    assert 600 < sum(want) < 2400
    assert meet(cases) == want


def test_views_of_one_projection(meet):
    b, hq, hkv, n, d = 16, 28, 4, 32768, 128
    wide = (hq + 2 * hkv) * d
    base = 1 << 40
    at = {"q": (base, n * wide, d, wide, hq), "k": (base + 2 * hq * d, n * wide, d, wide, hkv), "v": (base + 2 * (hq + hkv) * d, n * wide, d, wide, hkv)}
    at["heads first"] = (base, d, b * n * d, b * d, hq)    # other strides inside the same memory
    for x, y in itertools.product(at, at):
        if "heads first" in (x, y):
            assert meet([(at[x], at[y], b, n, d, 2)]) == [True]
        else:
            assert meet([(at[x], at[y], b, n, d, 2)]) == [x == y], (x, y)
    apart = (base + 2 * b * n * wide, hq * n * d, n * d, d, hq)
    assert meet([(at["q"], apart, b, n, d, 2), (apart, at["v"], b, n, d, 2)]) == [False, False]
    last = (base + 2 * (b * n * wide - d), hq * n * d, n * d, d, hq)          # its first row is the last of v
    assert meet([(at["v"], last, b, n, d, 2), (at["k"], last, b, n, d, 2), (last, at["v"], b, n, d, 2)]) == [True, False, True]
