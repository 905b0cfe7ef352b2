"""GPU: powattn_decode_paged_q4 where a row is cut into parts, whose partial results go through the workspace and a second kernel: a
workspace that holds NaN or old results, parts that have no chunk, graphs and streams.  Tolerances as in test_gpu_decode_q4.py."""
import numpy as np
import pytest
import torch

import test_gpu_decode_step_q4 as step
from around_util import values_of
from gpu_util import oracle_pattern
from oracle import powattn_oracle as orc
from paper_2503_03588_amd import binding as pa
from test_gpu_decode_q4 import make, run
from test_gpu_decode_step_q4 import Exact, Loop, f64, i32

pytestmark = pytest.mark.gpu

WIDE = pa.Pattern(64, 400, 1, 0)                           # a window over the whole cache
STRIDE = 40                                                # its row has 40 chunks: five rounds of a workgroup's wavefronts


def parts(pat, b, hq, hkv, d, stride):
    """parts of a row, from the workspace's size (that of one part, and less than one more for the alignment)"""
    one = b * hq * (d + 2) * 4
    return pa.decode_paged_q4_workspace_bytes(pat, b, hq, hkv, d, stride * pat.block) // one


def poisoned(b, hq, hkv, d, byte=255):
    return torch.full((pa.decode_paged_q4_workspace_bytes(WIDE, b, hq, hkv, d, STRIDE * 64),), byte, dtype=torch.uint8, device="cuda")


def verify(q, flat, lens, o, lse):
    k, v = flat
    for i, n in enumerate(lens):
        if n == 0:
            assert (o[i] == 0).all() and (lse[i] == -np.inf).all()
            continue
        want, want_lse = orc.decode(q[i: i + 1].double().numpy(), k[i: i + 1, :, :n], v[i: i + 1, :, :n], [n], oracle_pattern(WIDE))
        tol = 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -12 * np.abs(v[i, :, :n]).max()
        assert (np.abs(o[i] - want[0]) <= tol).all(), (i, n)
        assert (np.abs(lse[i] - want_lse[0]) <= 2.0 ** -13).all(), (i, n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 2), (14, 2), (16, 1)])
def test_whatever_the_workspace_holds(hq, hkv, d):
    lens = [2560, 1, 17 * 64, 0, 700, 65]                  # most parts of most rows have no chunk
    b = len(lens)
    assert parts(WIDE, b, hq, hkv, d, STRIDE) >= 2
    q, cache, table, flat = make(WIDE, b, hq, hkv, d, lens, seed=hq + d, capacity=STRIDE * 64)
    ws = poisoned(b, hq, hkv, d)
    first = run(WIDE, q, cache, table, lens, workspace=ws)
    verify(q, flat, lens, *first)
    for byte in (0, 127, 255, None):                       # None: as the call before has left it
        if byte is not None:
            ws.fill_(byte)
        assert all(np.array_equal(x, y) for x, y in zip(first, run(WIDE, q, cache, table, lens, workspace=ws)))
    lens[0] = 100                                          # (results of the longer row are still there)
    verify(q, flat, lens, *run(WIDE, q, cache, table, lens, workspace=ws))


@pytest.fixture
def wide(monkeypatch):
    monkeypatch.setattr(step, "PAT", WIDE)


def filled(batch, seed, lens, share=None):
    """a loop whose sequences hold `lens` tokens, and what they are"""
    loop, exact = Loop(batch, STRIDE, seed), Exact(batch)
    assert parts(WIDE, batch, step.HQ, step.HKV, step.D, STRIDE) >= 2
    if share is not None:
        loop.ws = share
    loop.ws.fill_(255)
    q, k, v = loop.attend(loop.project(max(lens)), i32(*lens))
    exact.add(k, v, lens)
    return loop, exact


def outputs(batch):
    return torch.empty((batch, step.HQ, step.D), dtype=torch.bfloat16, device="cuda"), torch.empty((batch, step.HQ), device="cuda")


def test_replayed_from_graphs_that_share_a_workspace(wide):
    lens, one = [1500, 3, 1087], i32(1, 1, 1)
    a = filled(3, 2, lens)
    both = [a, filled(3, 3, lens[::-1], share=a[0].ws)]
    graphs = []
    for loop, exact in both:
        x, (o, lse) = loop.project(1), outputs(3)
        q, k, v = loop.step(x, one, o, lse)
        exact.add(k, v, [1] * 3)
        exact.check(q, o, lse)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q, k, v = loop.step(x, one, o, lse)
        graphs.append((g, q, k, v, o, lse, x))
    for i in range(4):
        for (loop, exact), (g, q, k, v, o, lse, x) in zip(both, graphs):
            if i % 2:
                loop.ws.fill_(255)
            x.copy_(loop.project(1))
            g.replay()
            torch.cuda.synchronize()
            exact.add(k, v, [1] * 3)
            exact.check(q, o, lse)
            eager = pa.decode_paged_q4(WIDE, q[:, :, 0].contiguous(), loop.cache, loop.table, loop.held, workspace=loop.ws)
            assert torch.equal(eager[0], o) and torch.equal(eager[1], lse)


def test_two_calls_at_once(wide):
    lens = [1500, 5, 0, 1200]
    both, out = [filled(4, 6, lens), filled(4, 7, lens)], []
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(3):
        for (loop, exact), s in zip(both, streams):
            with torch.cuda.stream(s):
                o, lse = outputs(4)
                out.append((exact, *loop.step(loop.project(1), i32(1, 1, 1, 1), o, lse), o, lse))
    torch.cuda.synchronize()
    for exact, q, k, v, o, lse in out:
        exact.add(k, v, [1] * 4)
        exact.check(q, o, lse)


def test_as_the_decode_step_over_bf16_pages():
    # The bf16 step rounds every weight to bf16, off by 2^-8 of it at most, this one by 2^-17; scores and sums as in
    # test_gpu_decode_q4.py, twice; half a step of the output on either side.  All of it relative to the row's sum of p |v|.
    pat, b, hq, hkv, d = pa.Pattern(128, 4, 1), 4, 16, 4, 128
    lens = [1500, 129, 128, 3500]
    q, cache, table, (k, v) = make(pat, b, hq, hkv, d, lens, 15)
    pages = [torch.from_numpy(np.nan_to_num(values_of(cache[i].numpy(), cache[2 + i].numpy()))).bfloat16().cuda() for i in range(2)]
    t, n = torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = pa.decode_paged(pat, q.cuda(), *pages, t, n)
    o4, lse4 = run(pat, q, cache, table, lens)
    for i, m in enumerate(lens):
        size, _ = orc.decode(q[i: i + 1].double().numpy(), k[i: i + 1, :, :m], np.abs(v[i: i + 1, :, :m]), [m], oracle_pattern(pat))
        tol = 2.0 ** -7 * np.abs(o4[i]) + (2.0 ** -8 + 2.0 ** -17 + 2.0 ** -12) * size[0]
        assert (np.abs(f64(o)[i] - o4[i]) <= tol).all(), i
        assert 2.0 ** -8 * size[0].max() < 0.25 * np.sqrt((o4[i] ** 2).mean())             # (a fraction of a typical output)
    assert np.abs(f64(lse) - lse4).max() <= 2.0 ** -12
