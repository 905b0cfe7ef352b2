"""GPU: rows into the 4-bit cache and out of it.  The format is exact: what is stored equals the definition in 64 bits, code for
code, and what is loaded equals what the codes stand for."""
import numpy as np
import pytest
import torch

from around_util import codes_of, expand, shrink, tables, values_of
from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu


def rows(b, h, n, d, seed, layout="contiguous"):
    gen = torch.Generator().manual_seed(seed)
    if layout == "fused":
        whole = torch.randn((b, n, 3 * h * d), generator=gen).bfloat16()
        return whole[..., h * d: 2 * h * d].unflatten(2, (-1, d)).transpose(1, 2)
    if layout == "odd":
        whole = torch.randn((b, n, h * d + 5), generator=gen).bfloat16()
        return whole[..., 3: 3 + h * d].unflatten(2, (-1, d)).transpose(1, 2)
    if layout == "broadcast":
        return torch.randn((b, 1, n, d), generator=gen).bfloat16().expand(-1, h, -1, -1)
    return torch.randn((b, h, n, d), generator=gen).bfloat16()


def on_gpu(t):
    flat = torch.empty(0, dtype=t.dtype).set_(t.untyped_storage()).cuda()
    return flat.as_strided(t.shape, t.stride(), t.storage_offset())


def f64(t):
    return t.double().cpu().numpy()


def garbage(pat, n_pages, h, d, seed):
    cache = pa.cache_q4(pat, n_pages, h, d)
    gen = torch.Generator("cuda").manual_seed(seed)
    for t in cache:
        t.random_(0, 256, generator=gen)
    return cache


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,h,n,block,layout", [
    (1, 1, 1, 64, "contiguous"), (3, 2, 1, 64, "fused"), (2, 3, 77, 64, "odd"), (4, 2, 130, 128, "fused"), (2, 1, 65, 256, "broadcast"),
    (5, 8, 700, 64, "contiguous"), (2, 8, 2100, 192, "fused"),
])
def test_store_and_load(d, b, h, n, block, layout):
    pat = pa.Pattern(block, 4, 1)
    rng = np.random.default_rng(b * n + d)
    start, length = rng.integers(0, 3 * block, size=b), rng.integers(0, n + 1, size=b)
    length[0] = n
    stride = -(-(3 * block + n) // block)
    n_pages = b * stride + 3
    order = rng.permutation(n_pages)
    table, slots, _, _ = tables(block, start, length, n, order[b * stride:], n_pages, order[: b * stride].reshape(b, stride))
    for i in range(b):                                      # (more free pages than the three are not needed: fill in by hand)
        table[i] = order[i * stride: (i + 1) * stride]
        for r in range(int(length[i])):
            blk, off = divmod(int(start[i]) + r, block)
            slots[i, r] = table[i, blk] * block + off
    cache = garbage(pat, n_pages, h, d, 1)
    before = [t.cpu().numpy() for t in cache]
    k, v = rows(b, h, n, d, 2, layout), rows(b, h, n, d, 3, "fused")
    d_slots = torch.tensor(slots, dtype=torch.int32, device="cuda")
    pa.cache_store_q4(pat, on_gpu(k), on_gpu(v), cache, d_slots)
    after = [t.cpu().numpy() for t in cache]
    page, off = slots // block, slots % block
    there = slots >= 0
    for x, data, scale, was, was_scale in ((k, after[0], after[2], before[0], before[2]), (v, after[1], after[3], before[1], before[3])):
        code, sc = shrink(f64(x).transpose(0, 2, 1, 3)[there])                  # [tokens, h, d]
        assert np.array_equal(codes_of(data[page[there], :, off[there]]), code)
        assert np.array_equal(scale[page[there], :, :, off[there]], sc)
        was[page[there], :, off[there]] = data[page[there], :, off[there]]      # nothing else has changed
        was_scale[page[there], :, :, off[there]] = scale[page[there], :, :, off[there]]
        assert np.array_equal(was, data) and np.array_equal(was_scale, scale)

    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    out = [torch.full((b, h, n, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pa.cache_load_q4(pat, cache, i32(table), n, start=i32(start), length=i32(length), k=out[0], v=out[1])
    for x, got in ((k, out[0]), (v, out[1])):
        want = expand(*shrink(f64(x)))
        keep = np.broadcast_to(there[:, None], got.shape[:3])
        assert np.array_equal(f64(got)[keep], want[keep]) and (f64(got)[~keep] == 9.0).all()


def test_every_bf16_value_as_a_groups_largest():
    # one group for each of the 65536 bit patterns: the value itself, and 31 fractions of it of either sign
    pat, d = pa.Pattern(64, 4, 1), 64
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    part = torch.linspace(-1, 1, 31)
    x = torch.cat([bits[:, None].float(), bits[:, None].float() * part], 1).bfloat16()          # [65536, 32]
    k = x.view(1, 1, 32768, 64)
    cache = pa.cache_q4(pat, 512, 1, d)
    slots = torch.arange(32768, dtype=torch.int32, device="cuda").view(1, -1)
    pa.cache_store_q4(pat, k.cuda(), k.flip(2).contiguous().cuda(), cache, slots)
    kd, _, ks, _ = (t.cpu().numpy() for t in cache)
    with np.errstate(invalid="ignore"):
        code, scale = shrink(f64(k)[0, 0])
    assert np.array_equal(codes_of(kd.reshape(32768, 32)), code)
    assert np.array_equal(ks.transpose(0, 1, 3, 2).reshape(32768, 2), scale)
    table = torch.arange(512, dtype=torch.int32, device="cuda").view(1, -1)
    got, _ = pa.cache_load_q4(pat, cache, table, 32768)
    assert np.array_equal(f64(got)[0, 0], expand(code, scale), equal_nan=True)


def test_every_code_and_scale_is_loaded():
    pat = pa.Pattern(64, 4, 1)
    cache = pa.cache_q4(pat, 256, 1, 64)
    cache.k[:] = torch.arange(256, dtype=torch.uint8, device="cuda").repeat_interleave(32).view(256, 32)[:, None, None]
    cache.v[:] = cache.k
    cache.k_scale[:] = torch.arange(256, dtype=torch.uint8, device="cuda")[None, None, None].expand(256, 1, 2, 256)[..., :64]
    cache.v_scale[:] = torch.arange(192, 256, dtype=torch.uint8, device="cuda")
    table = torch.arange(256, dtype=torch.int32, device="cuda").view(1, -1)
    k, v = pa.cache_load_q4(pat, cache, table, 256 * 64)
    for got, data, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want = values_of(data.cpu().numpy(), scale.cpu().numpy()).reshape(1, 1, 256 * 64, 64)
        big = np.abs(want) >= 2.0 ** 128                    # codes that the store never writes: beyond bf16's numbers
        with np.errstate(invalid="ignore"):
            want = np.where(big, np.sign(want) * np.inf, want)
        assert np.array_equal(f64(got), want, equal_nan=True)


def test_slots_outside_the_pool_are_skipped_and_pages_clamped():
    pat = pa.Pattern(64, 4, 1)
    cache = garbage(pat, 3, 2, 128, 5)
    before = [t.clone() for t in cache]
    k = rows(1, 2, 4, 128, 6).cuda()
    slots = torch.tensor([[-1, 192, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    pa.cache_store_q4(pat, k, k, cache, slots)
    assert all(torch.equal(a, b) for a, b in zip(cache, before))
    lo, hi = (pa.cache_load_q4(pat, cache, torch.tensor([[p]], dtype=torch.int32, device="cuda"), 64) for p in (0, 2))
    for page, want in ((-7, lo), (3, hi), (2 ** 31 - 1, hi)):
        got = pa.cache_load_q4(pat, cache, torch.tensor([[page]], dtype=torch.int32, device="cuda"), 64)
        assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16))
        assert torch.equal(got[1].view(torch.int16), want[1].view(torch.int16))


def test_lengths_beyond_the_table():
    pat = pa.Pattern(64, 4, 1)
    cache = pa.cache_q4(pat, 4, 1, 64)
    table = torch.tensor([[1, 2], [3, 0]], dtype=torch.int32, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out = [torch.full((2, 1, 200, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pa.cache_load_q4(pat, cache, table, 200, start=i32(100, 5000), length=i32(1000, 3), k=out[0], v=out[1])
    for t in out:
        assert (t[0, 0, :28] == 0).all() and (t[0, 0, 28:] == 9).all() and (t[1] == 9).all()


def test_a_pool_beyond_32_bit_offsets():
    # 4.4 GB of pages: the last page lies behind 2^32 bytes
    pat, h, d = pa.Pattern(1024, 4, 1), 8, 128
    n_pages = 8400
    cache = pa.cache_q4(pat, n_pages, h, d)
    assert cache.k.numel() > 2 ** 32
    k, v = rows(1, h, 1000, d, 7), rows(1, h, 1000, d, 8)
    slots = ((n_pages - 1) * 1024 + 10 + torch.arange(1000, dtype=torch.int32, device="cuda")).view(1, -1).int()
    pa.cache_store_q4(pat, k.cuda(), v.cuda(), cache, slots)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    start = torch.tensor([10], dtype=torch.int32, device="cuda")
    got = pa.cache_load_q4(pat, cache, table, 1000, start=start)
    for x, y in ((k, got[0]), (v, got[1])):
        assert np.array_equal(f64(y), expand(*shrink(f64(x))))
    assert not cache.k[: n_pages - 1].any() and not cache.v_scale[: n_pages - 1].any()
