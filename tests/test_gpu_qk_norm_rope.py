"""GPU: powattn_qk_norm_rope and its gradients against the formulas in 64 bits.

Tolerances.  With u the row before the rotation, a component of fp32 arithmetic is off by at most 2^-19 (|u_i| + |u_j|) of its
pair: the sum of squares of a lane's 16 components and three exchanges (20 roundings, half of them under the root), root, quotient,
two products, cosine and sine (2 units each, and 2^-26 of a turn from the reduced angle), two products and a sum: below 32
roundings of 2^-24.  A gradient has one more such sum: 2^-18 of what it is a sum of.  dw sums at most 40 heads of one token in a
chain, then at most 6 + 4 + 32 + 32 further terms, each 20 roundings off: 160 * 2^-24 of the sum of magnitudes.  Outputs in bf16 are
rounded once: 2^-8 of their value (half a step)."""
import numpy as np
import pytest
import torch

from around_util import norm_rope, norm_rope_grad
from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def inputs(dtype, b, hq, hkv, n, d, rot, seed, layout="fused", scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    t = TYPES[dtype]
    new = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
    if layout == "fused":                                   # views of a projection's output
        whole = (new(b, n, (hq + 2 * hkv) * d) * scale).to(t)
        q, k, _ = (x.unflatten(2, (-1, d)).transpose(1, 2) for x in whole.split([hq * d, hkv * d, hkv * d], 2))
    elif layout == "contiguous":
        q, k = (new(b, hq, n, d) * scale).to(t), (new(b, hkv, n, d) * scale).to(t)
    elif layout == "odd":                                   # rows an odd number of components apart, an odd offset
        whole = (new(b, n, (hq + hkv) * d + 3) * scale).to(t)
        q = whole[..., 1: 1 + hq * d].unflatten(2, (-1, d)).transpose(1, 2)
        k = whole[..., 1 + hq * d: 1 + (hq + hkv) * d].unflatten(2, (-1, d)).transpose(1, 2)
    elif layout == "broadcast":                             # one sequence for the whole batch
        q, k = new(1, hq, n, d).to(t).expand(b, -1, -1, -1), new(1, hkv, n, d).to(t).expand(b, -1, -1, -1)
    elif layout == "reversed":                              # heads slowest in memory
        q, k = (new(h, n, b, d).to(t).permute(2, 0, 1, 3) for h in (hq, hkv))
    w = [(1 + 0.3 * new(d)).to(t) for _ in range(2)]
    inv_freq = (1e6 ** (-torch.arange(0, rot, 2).double() / rot)).float() if rot else None
    return q, k, w, inv_freq


def on_gpu(t):
    """the same strides on the GPU"""
    if t is None:
        return None
    storage = t.untyped_storage()
    flat = torch.empty(0, dtype=t.dtype).set_(storage).cuda()
    return flat.as_strided(t.shape, t.stride(), t.storage_offset())


def f64(t):
    return t.double().cpu().numpy()


def close(got, want, big, dtype, bits):
    tol = HALF_STEP[dtype] * np.abs(want) + 2.0 ** -bits * big + 1e-37
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)


def pair_size(u, rot, interleaved):
    from around_util import pairs
    big = np.abs(u)
    if rot:
        i, j = pairs(rot, interleaved)
        s = big[..., i] + big[..., j]
        big[..., i] = s
        big[..., j] = s
    return big


CASES = [
    # dtype, b, hq, hkv, n, d, rot, interleaved, layout, start, q_len
    ("bf16", 1, 1, 1, 1, 128, 128, False, "fused", [0], None),
    ("bf16", 2, 4, 2, 33, 128, 128, False, "fused", [0, 1000003], None),
    ("bf16", 3, 28, 4, 1, 128, 128, False, "fused", [5, 65535, 131071], None),
    ("bf16", 2, 5, 1, 100, 64, 64, False, "contiguous", [7, 0], [100, 31]),
    ("f32", 2, 4, 2, 70, 64, 32, True, "fused", [999983, 12], [0, 70]),
    ("f32", 1, 7, 3, 65, 128, 64, False, "odd", [400000], None),
    ("bf16", 2, 3, 2, 41, 128, 96, True, "odd", [1, 2], [40, 41]),
    ("f32", 2, 2, 2, 130, 128, 16, False, "reversed", [0, 9], None),
    ("bf16", 1, 40, 8, 257, 64, 48, False, "reversed", [3], None),
    ("bf16", 2, 2, 1, 20, 128, 0, False, "contiguous", [0, 0], None),
    ("f32", 3, 2, 1, 20, 64, 64, True, "broadcast", [0, 50, 2000000000], None),
    ("f32", 1, 1, 1, 600, 64, 64, False, "contiguous", [123456], [600]),
]


@pytest.mark.parametrize("dtype,b,hq,hkv,n,d,rot,inter,layout,start,q_len", CASES)
def test_forward(dtype, b, hq, hkv, n, d, rot, inter, layout, start, q_len):
    q, k, w, inv = inputs(dtype, b, hq, hkv, n, d, rot, 11, layout)
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q_out = torch.full((b, hq, n, d), 7.0, dtype=TYPES[dtype], device="cuda")
    k_out = torch.full((b, hkv, n, d), 7.0, dtype=TYPES[dtype], device="cuda")
    pa.qk_norm_rope(on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), None if inv is None else inv.cuda(), q_start=i32(start),
                    q_len=i32(q_len), eps=1e-5, interleaved=inter, q_out=q_out, k_out=k_out)
    there = np.arange(n) < np.array(q_len if q_len else [n] * b)[:, None]
    for x, wt, out in ((q, w[0], q_out), (k, w[1], k_out)):
        y, u = norm_rope(f64(x), f64(wt), None if inv is None else inv.numpy(), start, 1e-5, inter)
        keep = np.broadcast_to(there[:, None], out.shape[:3])
        got = f64(out)
        assert (got[~keep] == 7.0).all()                    # rows behind a sequence's last one
        close(got[keep], y[keep], pair_size(u, rot, inter)[keep], dtype, 19)


@pytest.mark.parametrize("dtype,b,hq,hkv,n,d,rot,inter,layout,start,q_len", CASES)
def test_gradients(dtype, b, hq, hkv, n, d, rot, inter, layout, start, q_len):
    q, k, w, inv = inputs(dtype, b, hq, hkv, n, d, rot, 12, layout)
    gen = torch.Generator().manual_seed(13)
    dy = [torch.randn(x.shape, generator=gen).to(TYPES[dtype]) for x in (q, k)]
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    there = np.arange(n) < np.array(q_len if q_len else [n] * b)[:, None]
    for g in dy:                                            # what must not be read holds no numbers
        g.transpose(1, 2)[torch.from_numpy(~there)] = float("nan")
    given = {}
    if layout in ("fused", "odd"):                          # into the gradient of the projections' output
        extra = 2 * hkv * d if layout == "fused" else hkv * d + 3
        whole = torch.full((b, n, hq * d + extra), 7.0, dtype=TYPES[dtype], device="cuda")
        at = 0 if layout == "fused" else 1
        given = {"dq": whole[..., at: at + hq * d].unflatten(2, (-1, d)).transpose(1, 2),
                 "dk": whole[..., at + hq * d: at + (hq + hkv) * d].unflatten(2, (-1, d)).transpose(1, 2)}
    got = pa.qk_norm_rope_backward(on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), None if inv is None else inv.cuda(), dy[0].cuda(),
                                   dy[1].cuda(), q_start=i32(start), q_len=i32(q_len), eps=1e-5, interleaved=inter, **given)
    again = pa.qk_norm_rope_backward(on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), None if inv is None else inv.cuda(),
                                     dy[0].cuda(), dy[1].cuda(), q_start=i32(start), q_len=i32(q_len), eps=1e-5, interleaved=inter)
    for x, wt, g, dx, dw, dw2 in ((q, w[0], dy[0], got[0], got[2], again[2]), (k, w[1], dy[1], got[1], got[3], again[3])):
        want, want_w, (big, big_w) = norm_rope_grad(f64(x), f64(wt), None if inv is None else inv.numpy(), start, 1e-5, inter,
                                                    np.nan_to_num(f64(g)), there)
        keep = np.broadcast_to(there[:, None], dx.shape[:3])
        if given:
            assert (f64(dx)[~keep] == 7.0).all()
        else:
            assert (f64(dx)[~keep] == 0.0).all()
        close(f64(dx)[keep], want[keep], big[keep], dtype, 18)
        assert (np.abs(f64(dw) - want_w) <= 160 * 2.0 ** -24 * big_w + 1e-37).all()
        assert torch.equal(dw, dw2)                         # the sums have a fixed order
    if given:
        rest = whole[..., (hq + hkv) * d + at:]
        assert (rest == 7.0).all()


def test_gradients_against_differences():
    b, hq, hkv, n, d, rot, start = 2, 3, 1, 9, 64, 32, [100, 5000]
    q, k, w, inv = inputs("f32", b, hq, hkv, n, d, rot, 21)
    gen = torch.Generator().manual_seed(22)
    dy = [torch.randn(x.shape, generator=gen) for x in (q, k)]
    s = torch.tensor(start, dtype=torch.int32, device="cuda")
    got = pa.qk_norm_rope_backward(on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), inv.cuda(), dy[0].cuda(), dy[1].cuda(), q_start=s)
    rng = np.random.default_rng(23)
    for x, wt, g, dx, dw in ((q, w[0], dy[0], got[0], got[2]), (k, w[1], dy[1], got[1], got[3])):
        f = lambda xx, ww: (norm_rope(xx, ww, inv.numpy(), start, 1e-6, False)[0] * f64(g)).sum()  # noqa: E731
        for _ in range(3):
            vx, vw, h = rng.standard_normal(x.shape), rng.standard_normal(d), 1e-5
            along = (f(f64(x) + h * vx, f64(wt) + h * vw) - f(f64(x) - h * vx, f64(wt) - h * vw)) / (2 * h)
            mine = (f64(dx) * vx).sum() + (f64(dw) * vw).sum()
            # second-order differences: h^2 of a sum of this size, and the cancellation 2^-52 f / h
            size = np.abs(f64(dx) * vx).sum() + np.abs(f64(dw) * vw).sum()
            assert abs(along - mine) <= 1e-5 * size


def test_many_rows_fill_every_workgroup():
    # more token groups than workgroups: the gradients' workgroups walk on
    b, hq, hkv, n, d = 1, 16, 2, 20011, 64
    q, k, w, inv = inputs("bf16", b, hq, hkv, n, d, 64, 31)
    gen = torch.Generator().manual_seed(32)
    dy = [torch.randn(x.shape, generator=gen).to(torch.bfloat16) for x in (q, k)]
    args = (on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), inv.cuda())
    outs = pa.qk_norm_rope(*args)
    got = pa.qk_norm_rope_backward(*args, dy[0].cuda(), dy[1].cuda())
    for x, wt, g, out, dx, dw in ((q, w[0], dy[0], outs[0], got[0], got[2]), (k, w[1], dy[1], outs[1], got[1], got[3])):
        y, u = norm_rope(f64(x), f64(wt), inv.numpy(), [0], 1e-6, False)
        close(f64(out), y, pair_size(u, 64, False), "bf16", 19)
        want, want_w, (big, big_w) = norm_rope_grad(f64(x), f64(wt), inv.numpy(), [0], 1e-6, False, f64(g), np.ones((b, n), bool))
        close(f64(dx), want, big, "bf16", 18)
        assert (np.abs(f64(dw) - want_w) <= 160 * 2.0 ** -24 * big_w).all()


def test_rows_of_zeros_and_without_numbers():
    b, hq, hkv, n, d = 1, 2, 1, 6, 128
    q, k, w, inv = inputs("f32", b, hq, hkv, n, d, 64, 41, "contiguous")
    q[0, 0, 2] = 0
    q[0, 1, 3, 5] = float("nan")
    q[0, 1, 4, 100] = float("inf")
    out, _ = pa.qk_norm_rope(q.cuda(), k.cuda(), w[0].cuda(), w[1].cuda(), inv.cuda())
    assert (out[0, 0, 2] == 0).all() and out[0, 1, 3].isnan().all()
    assert out[0, 1, 4, 100].isnan() and torch.isfinite(out[0, 1, 4, 64:100]).all()        # inf / inf; the others are 0
    assert torch.isfinite(out[0, 0]).all() and torch.isfinite(out[0, 1, [0, 1, 2, 5]]).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 16384), ("f32", 9000)])
def test_a_large_call_is_its_parts(dtype, n):
    # beyond 128 MB the outputs are written past the caches: the same bits as from calls on parts of the rows
    b, hq, hkv, d = 1, 18, 2, 128
    q, k, w, inv = inputs(dtype, b, hq, hkv, n, d, d, 51)
    gen = torch.Generator("cuda").manual_seed(52)
    q, k, w, inv = on_gpu(q), on_gpu(k), [x.cuda() for x in w], inv.cuda()
    dy = [torch.randn(x.shape, generator=gen, device="cuda").to(TYPES[dtype]) for x in (q, k)]
    assert 2 * (q.numel() + k.numel()) * q.element_size() > 128 << 20
    outs, grads = pa.qk_norm_rope(q, k, *w, inv), pa.qk_norm_rope_backward(q, k, *w, inv, *dy)
    for lo, hi in ((0, 3000), (3000, 3001), (n - 2500, n)):
        start = torch.tensor([lo], dtype=torch.int32, device="cuda")
        parts = [x[:, :, lo:hi] for x in (q, k)]
        got = pa.qk_norm_rope(*parts, *w, inv, q_start=start)
        assert all(torch.equal(a[:, :, lo:hi], x) for a, x in zip(outs, got))
        got = pa.qk_norm_rope_backward(*parts, *w, inv, *(x[:, :, lo:hi].contiguous() for x in dy), q_start=start)
        assert all(torch.equal(a[:, :, lo:hi], x) for a, x in zip(grads[:2], got[:2]))


def test_a_batch_without_rows():
    q, k, w, inv = inputs("bf16", 2, 3, 1, 40, 64, 64, 61)
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    args = (on_gpu(q), on_gpu(k), w[0].cuda(), w[1].cuda(), inv.cuda())
    for t in pa.qk_norm_rope(*args, q_len=none):
        assert not t.any()
    nan = [torch.full(x.shape, float("nan"), dtype=torch.bfloat16, device="cuda") for x in (q, k)]
    for t in pa.qk_norm_rope_backward(*args, *nan, q_len=none):
        assert not t.any()
