"""GPU: how exactly powattn_decode_paged_q4 holds a row's weights.

A row of two tokens: the first has a key and a value of zeros, the second a score s and a value v, so that its weight is P = exp(s) and
the output v P / (1 + P).  P is multiplied in two bf16 parts, each rounded to the nearest: what the first leaves is at most 2^-8 of P's power of
two, half a step of that is 2^-17 of P at most, to either side.  (Two parts that are cut: too small by up to 2^-15.)  The scores are sums of two products, exact in fp32; scale, difference, exp2 and
the quotient are ten roundings of 2^-24 on numbers below 8: 2^-18.  The output's own rounding is half a step."""
import numpy as np
import pytest
import torch

from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu


def half_step(x):
    """half the distance between the bf16 numbers around x"""
    return 2.0 ** (np.floor(np.log2(np.abs(x))) - 8)


def cut(x):
    return (np.float32(x).view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)


def queries(n, seed):
    """Pairs of components whose row has a weight with a long tail of ones, and one of the outputs 1 / 1.5 times P / (1 + P) just above
    a border of the rounding: nearer to it than a weight of two cut parts would be off, further than the tolerance."""
    rng = np.random.default_rng(seed)
    q = torch.from_numpy(np.stack([-rng.uniform(0.1, 4, 1 << 21), rng.uniform(0, 2 ** -7, 1 << 21)], -1)).bfloat16().double().numpy()
    p = np.exp(q.sum(-1))
    top = cut(p).astype(np.float64)
    low = (p - top - cut(p - top)) / p                     # what two cut parts leave out
    keep = np.zeros(len(p), bool)
    for v in (1.0, 1.5):
        o = v * p / (1 + p)
        step = 2 * half_step(o)
        above = ((o / step - 0.5) % 1) * step / o          # the border below, relative to o
        keep |= (above > 2.0 ** -16 + 2.0 ** -18 + 2.0 ** -21) & (above + 2.0 ** -20 < low)
    assert keep.any()
    return q[keep][np.arange(n) % keep.sum()]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [4, 8, 16])
def test_weights_are_rounded_to_the_nearest(hq, d):
    pat, b = pa.Pattern(64, 1, 0), 8
    two = queries(b * hq, seed=hq + d).reshape(b, hq, 2)
    q = torch.zeros((b, hq, d), dtype=torch.bfloat16)
    q[..., [0, 1]] = torch.from_numpy(two).bfloat16()
    k, v = (torch.zeros((b, 1, 2, d), dtype=torch.bfloat16) for _ in range(2))
    k[:, :, 1, :2] = 1.0
    v[:, :, 1] = torch.tensor([1.0, 1.5, -3.0, 4.0]).repeat(d // 4).bfloat16()
    cache = pa.cache_q4(pat, b, 1, d)
    table = torch.arange(b, dtype=torch.int32, device="cuda").view(b, 1)
    pa.cache_store_q4(pat, k.cuda(), v.cuda(), cache, table * 64 + torch.arange(2, dtype=torch.int32, device="cuda"))
    o, _ = pa.decode_paged_q4(pat, q.cuda(), cache, table, torch.full((b,), 2, dtype=torch.int32, device="cuda"), softmax_scale=1.0)
    p = np.exp(two.sum(-1))[..., None]
    want = p / (1 + p) * v[:, :, 1].double().numpy()
    off = np.abs(o.double().cpu().numpy() - want)
    assert (off <= half_step(want) + (2.0 ** -17 + 2.0 ** -18) * np.abs(want)).all(), (off / np.abs(want)).max() * 2 ** 16
