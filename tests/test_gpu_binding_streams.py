"""GPU: calls on another stream than the current one, which is busy meanwhile: what the call makes itself is made on its own stream, so that
a fill that waits behind the current stream's work does not come after the kernel."""
import pytest
import torch

from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu

PAT = pa.Pattern(64, 2, 1)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def new(*shape):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(sum(shape)), device="cuda").bfloat16()


def calls():
    b, hq, hkv, n, d = 2, 4, 2, 192, 64
    q, k, w, inv, lens = new(b, hq, n, d), new(b, hkv, n, d), new(d), torch.rand(16, device="cuda"), i32(192, 50)
    cnt, idx, _ = pa.mask_build(PAT, n)
    cache = pa.cache_q4(PAT, 6, hkv, d)
    table = i32(*range(6)).view(2, 3)
    slots = table.repeat_interleave(64, 1) * 64 + torch.arange(64, device="cuda").repeat(3).int()
    pa.cache_store_q4(PAT, k, k, cache, slots)
    q1, start, more, free = q[:, :, 0].contiguous(), i32(182, 40), i32(10, 10), i32(3, 4, 5)
    return {
        "varlen": lambda **kw: pa.prefill_varlen(PAT, cnt, idx, q, k, k, lens, **kw),
        "rope": lambda **kw: pa.qk_norm_rope(q, k, w, w, inv, q_len=lens, **kw),
        "rope_grad": lambda **kw: pa.qk_norm_rope_backward(q, k, w, w, inv, q, k, q_len=lens, **kw),
        "load": lambda **kw: pa.cache_load_q4(PAT, cache, table, n, length=lens, **kw),
        "decode_q4": lambda **kw: pa.decode_paged_q4(PAT, q1, cache, table, lens, **kw),
        "decode": lambda **kw: pa.decode(PAT, q1, k, k, lens, **kw),
        "tables": lambda **kw: pa.page_tables(PAT, start, more, free, table, 6, 10, **kw),
    }


@pytest.mark.parametrize("name", ["varlen", "rope", "rope_grad", "load", "decode_q4", "decode", "tables"])
@pytest.mark.parametrize("how", ["stream", "handle"])
def test_beside_a_busy_stream(name, how):
    call = calls()[name]
    want = [t.clone() for t in call()]
    side, big = torch.cuda.Stream(), torch.randn(8192, 8192, device="cuda").bfloat16()
    torch.cuda.synchronize()
    for _ in range(20):
        big = big @ big
    got = call(stream=side if how == "stream" else side.cuda_stream)
    side.synchronize()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
