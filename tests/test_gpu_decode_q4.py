"""GPU: powattn_decode_paged_q4 against the oracle on the keys and values that the cache stands for.

Tolerances.  Scores: products of bf16 numbers summed in fp32, 128 roundings of 2^-24 on sums below 64 here, 2^-11 at worst and
2^-18 as they fall (the roundings have either sign); the same for the log-sum-exp, which is held to 2^-13.  Outputs: half a
bf16 step, 2^-8 of the value, and weights that are off by twice the scores' error and 2^-16 (P in two parts), of the
largest |v|: 2^-12 of it."""
import numpy as np
import pytest
import torch

from around_util import values_of
from gpu_util import oracle_pattern
from oracle import powattn_oracle as orc
from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu


def make(pat, b, hq, hkv, d, kv_len, seed, n_extra=2, capacity=None):
    """q, the cache (CPU), the table and the float64 caches [b,Hkv,cap,D]; rows that nobody attends hold no numbers"""
    rng = np.random.default_rng(seed)
    stride = max(1, -(-max(capacity or 0, *kv_len) // pat.block))
    n_pages = b * stride + n_extra
    data, scale = (n_pages, hkv, pat.block, d // 2), (n_pages, hkv, d // 32, pat.block)
    # every code, scales 2^-4 .. 2^-1: components of 0.2 to 1.5 in the mean square
    cache = [torch.from_numpy(rng.integers(*r, size=s, dtype=np.uint8)) for r, s in (((0, 256), data), ((0, 256), data),
                                                                                    ((123, 127), scale), ((123, 127), scale))]
    table = rng.permutation(n_pages)[: b * stride].reshape(b, stride)
    vals = [values_of(cache[i].numpy(), cache[2 + i].numpy()) for i in range(2)]
    flat = [x[table].transpose(0, 2, 1, 3, 4).reshape(b, hkv, stride * pat.block, d) for x in vals]
    for i in range(b):                                     # behind the last token: NaN scales
        n = max(int(kv_len[i]), 0)
        for j in range(stride):
            lo = min(max(n - j * pat.block, 0), pat.block)
            for t in cache[2:]:
                t[int(table[i, j]), :, :, lo:] = 255
    for t in cache[2:]:
        for p in set(range(n_pages)) - set(table.reshape(-1).tolist()):
            t[p] = 255
    q = torch.from_numpy(rng.standard_normal((b, hq, d))).bfloat16()
    return q, cache, table, flat


def run(pat, q, cache, table, kv_len, **kw):
    o, lse = pa.decode_paged_q4(pat, q.cuda(), [t.cuda() for t in cache], torch.tensor(table, dtype=torch.int32, device="cuda"),
                                torch.tensor(kv_len, dtype=torch.int32, device="cuda"), **kw)
    return o.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()


def check(pat, b, hq, hkv, d, kv_len, seed, scale=0.0, **kw):
    q, cache, table, (k, v) = make(pat, b, hq, hkv, d, kv_len, seed, **kw)
    o, lse = run(pat, q, cache, table, kv_len, softmax_scale=scale)
    for i, n in enumerate(kv_len):
        if n <= 0:
            assert (o[i] == 0).all() and (lse[i] == -np.inf).all()
            continue
        want, want_lse = orc.decode(q[i: i + 1].double().numpy(), k[i: i + 1, :, :n], v[i: i + 1, :, :n], [n], oracle_pattern(pat),
                                    scale if scale > 0 else None)
        tol = 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -12 * np.abs(v[i, :, :n]).max()
        assert (np.abs(o[i] - want[0]) <= tol).all(), (i, n, np.abs(o[i] - want[0]).max())
        assert (np.abs(lse[i] - want_lse[0]) <= 2.0 ** -13).all(), (i, n, np.abs(lse[i] - want_lse[0]).max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (6, 2), (14, 2), (8, 1), (9, 1), (32, 2), (24, 8)])
def test_heads(d, hq, hkv):
    check(pa.Pattern(64, 2, 1), 3, hq, hkv, d, [700, 65, 1], seed=hq * d)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 16, 17, 63, 64, 65, 127, 128, 129, 1000, 1023, 4097])
def test_lengths(n):
    check(pa.Pattern(64, 4, 1), 2, 4, 2, 128, [n, max(n - 1, 1)], seed=n)
    check(pa.Pattern(128, 2, 0), 1, 8, 2, 64, [n], seed=n + 1)


@pytest.mark.parametrize("pat", [pa.Pattern(64, 0, 0), pa.Pattern(64, 5, 3, 0), pa.Pattern(128, 4, 1), pa.Pattern(192, 1, 2), pa.Pattern(256, 5, 1),
                                 pa.Pattern(1024, 2, 1)])
def test_patterns(pat):
    check(pat, 3, 8, 2, 128, [9000, 5 * pat.block + 1, 3 * pat.block], seed=pat.block)


def test_idle_places_of_a_batch():
    check(pa.Pattern(64, 4, 1), 6, 8, 2, 128, [0, 300, -4, 0, 5000, 1], seed=3)
    check(pa.Pattern(64, 4, 1), 2, 4, 1, 64, [0, 0], seed=4, capacity=70)
    q, cache, table, _ = make(pa.Pattern(64, 4, 1), 2, 4, 1, 128, [0, 100], 5)
    table[0] = -1                                          # an idle place has no pages
    o, lse = run(pa.Pattern(64, 4, 1), q, cache, table, [0, 100])
    assert (o[0] == 0).all() and (lse[0] == -np.inf).all() and np.isfinite(o[1]).all()


@pytest.mark.parametrize("b,hq,hkv,d", [(1, 32, 8, 128), (2, 28, 4, 128), (8, 8, 8, 64), (33, 16, 8, 128), (70, 32, 8, 128), (300, 4, 4, 64)])
def test_batches(b, hq, hkv, d):
    rng = np.random.default_rng(b)
    check(pa.Pattern(64, 4, 1), b, hq, hkv, d, [int(x) for x in rng.integers(1, 1500 if b > 8 else 9000, size=b)], seed=b)


def test_many_chunks():
    # a window over the whole cache: more chunks than the wavefronts of a workgroup, more passes than one
    check(pa.Pattern(64, 400, 1, 0), 1, 4, 1, 128, [20001], seed=7)
    check(pa.Pattern(64, 400, 1, 0), 2, 10, 1, 64, [20001, 700], seed=8)
    check(pa.Pattern(1024, 4, 1), 5, 8, 4, 128, [12000, 9999, 1, 1025, 4096], seed=9)
    check(pa.Pattern(64, 60, 1), 40, 8, 8, 64, [2000 + 37 * i for i in range(40)], seed=10)


def test_large_scores():
    # a softmax scale of 1: nearly one-hot rows
    check(pa.Pattern(64, 4, 1), 2, 4, 2, 128, [3000, 64], seed=11, scale=1.0 / 4)


def test_no_lse_and_outputs_given():
    pat = pa.Pattern(64, 4, 1)
    q, cache, table, _ = make(pat, 2, 4, 2, 128, [500, 900], 12)
    o, lse = run(pat, q, cache, table, [500, 900])
    o2, lse2 = run(pat, q, cache, table, [500, 900], want_lse=False)
    assert lse2 is None and np.array_equal(o, o2)
    mine = torch.empty((2, 4, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((pa.decode_paged_q4_workspace_bytes(pat, 2, 4, 2, 128, table.shape[1] * 64),), 255, dtype=torch.uint8, device="cuda")
    o3, _ = run(pat, q, cache, table, [500, 900], o=mine, workspace=ws)
    assert np.array_equal(o, o3) and np.array_equal(mine.double().cpu().numpy(), o)


def test_lengths_and_pages_outside_are_clamped():
    pat = pa.Pattern(64, 4, 1)
    q, cache, table, _ = make(pat, 1, 4, 2, 128, [640], 13)
    o, lse = run(pat, q, cache, table, [640])
    o2, lse2 = run(pat, q, cache, table, [100000])
    assert np.array_equal(o, o2) and np.array_equal(lse, lse2)
    n_pages = cache[0].shape[0]
    cache = [t.clone() for t in cache]
    for t in cache[2:]:
        t[:] = 120
    bad, good = table.copy(), table.copy()
    bad[0, 9], bad[0, 8] = n_pages + 5, -3
    good[0, 9], good[0, 8] = n_pages - 1, 0
    assert np.array_equal(run(pat, q, cache, bad, [640])[0], run(pat, q, cache, good, [640])[0])


@pytest.mark.parametrize("pat", [pa.Pattern(64, 2, 1), pa.Pattern(64, 400, 1, 0)], ids=["one workgroup", "several"])
def test_a_key_or_value_without_a_number(pat):
    for n in (200, 5000):
        q, cache, table, _ = make(pat, 2, 4, 2, 128, [n, n], 14)
        o, lse = run(pat, q, cache, table, [n, n])
        key = [t.clone() for t in cache]
        key[2][int(table[0, (n - 1) // 64]), 1, 2, 3] = 255                       # a key of sequence 0, KV head 1
        o1, lse1 = run(pat, q, key, table, [n, n])
        assert np.isnan(o1[0, 2:]).all() and np.isnan(lse1[0, 2:]).all()
        assert np.array_equal(o1[0, :2], o[0, :2]) and np.array_equal(o1[1], o[1]) and np.array_equal(lse1[1], lse[1])
        value = [t.clone() for t in cache]
        value[3][int(table[0, 0]), 0, 3, 60] = 255                                # components 96.. of a value, KV head 0
        o2, lse2 = run(pat, q, value, table, [n, n])
        assert np.isnan(o2[0, :2, 96:]).all() and np.array_equal(o2[0, :2, :96], o[0, :2, :96])
        assert np.array_equal(lse2, lse) and np.array_equal(o2[0, 2:], o[0, 2:])


def test_as_the_decode_step_over_bf16_pages():
    pat, b, hq, hkv, d = pa.Pattern(128, 4, 1), 4, 16, 4, 128
    lens = [3000, 129, 128, 7000]
    q, cache, table, _ = make(pat, b, hq, hkv, d, lens, 15)
    pages = [torch.from_numpy(np.nan_to_num(values_of(cache[i].numpy(), cache[2 + i].numpy()))).bfloat16().cuda() for i in range(2)]
    t, n = torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = pa.decode_paged(pat, q.cuda(), *pages, t, n)
    o4, lse4 = run(pat, q, cache, table, lens)
    # the bf16 step rounds P to bf16: up to 2^-9 of the largest |v| more, and half a step of the output on either side
    tol = 2.0 ** -7 * np.abs(o4) + (2.0 ** -9 + 2.0 ** -11) * 12
    assert (np.abs(o.double().cpu().numpy() - o4) <= tol).all()
    assert np.abs(lse.double().cpu().numpy() - lse4).max() <= 2.0 ** -12


def test_scores_are_summed_in_32_bits():
    # queries whose components differ by 2^13 and rows of one to three keys, whose log-sum-exp is hardly more than a score.  128
    # products of bf16 numbers, exact in fp32: 128 roundings of 2^-24 of the sum of magnitudes, and 2^-20 for exp, log and scale
    pat, b, hq, hkv, d = pa.Pattern(64, 2, 1), 24, 8, 2, 128
    lens = [1 + i % 3 for i in range(b)]
    q, cache, table, (k, v) = make(pat, b, hq, hkv, d, lens, 16)
    rng = np.random.default_rng(17)
    q = (q.double() * torch.from_numpy(2.0 ** -rng.integers(0, 14, size=q.shape))).bfloat16()
    _, lse = run(pat, q, cache, table, lens)
    for i, n in enumerate(lens):
        qi, ki = q[i].double().numpy(), k[i, :, :n].repeat(hq // hkv, 0)
        s = (qi[:, None] * ki).sum(-1) / np.sqrt(d)
        size = (np.abs(qi[:, None] * ki).sum(-1) / np.sqrt(d)).max(-1)
        want = np.log(np.exp(s - s.max(-1, keepdims=True)).sum(-1)) + s.max(-1)
        assert (np.abs(lse[i] - want) <= 2.0 ** -17 * size + 2.0 ** -20 * (1 + np.abs(want))).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(3, 1), (8, 1), (12, 2), (12, 1), (16, 1)])
def test_heads_of_a_row_in_several_parts(d, hq, hkv):
    check(pa.Pattern(64, 400, 1, 0), 2, hq, hkv, d, [5000, 1 + 64 * 9], seed=hq + d)


def test_pages_beyond_32_bit_offsets():
    pat, hq, hkv, d, n = pa.Pattern(1024, 2, 1), 8, 8, 128, 1500
    cache = pa.cache_q4(pat, 8400, hkv, d)
    assert cache.k.numel() > 2 ** 32
    gen = torch.Generator().manual_seed(18)
    k, v = (torch.randn((1, hkv, n, d), generator=gen).bfloat16().cuda() for _ in range(2))
    q = torch.randn((1, hq, d), generator=gen).bfloat16()
    table = torch.tensor([[8399, 8398]], dtype=torch.int32, device="cuda")
    pos = torch.arange(n, device="cuda")
    slots = (table[0, (pos // 1024)].long() * 1024 + pos % 1024).int().view(1, n)
    pa.cache_store_q4(pat, k, v, cache, slots)
    o, lse = pa.decode_paged_q4(pat, q.cuda(), cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    held = [t.double().cpu().numpy() for t in pa.cache_load_q4(pat, cache, table, n)]
    want, want_lse = orc.decode(q.double().numpy(), *held, [n], oracle_pattern(pat))
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * np.abs(held[1]).max()
    assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= 2.0 ** -13
