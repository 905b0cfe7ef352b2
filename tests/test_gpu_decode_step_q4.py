"""GPU: pages and slots, norm and rotation, the 4-bit cache and the decode step over it, one after the other as a serving loop
calls them: a padded batch of prompts, then one token after the other, eager and replayed from a graph; a further piece of a
prompt against the loaded cache.  Tolerances as in test_gpu_decode_q4.py."""
import numpy as np
import pytest
import torch

from around_util import expand, shrink
from gpu_util import oracle_pattern
from oracle import powattn_oracle as orc
from paper_2503_03588_amd import binding as pa

pytestmark = pytest.mark.gpu

PAT, HQ, HKV, D, ROT = pa.Pattern(64, 2, 1), 8, 2, 128, 64


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


class Loop:
    """What a serving program keeps for one layer."""

    def __init__(self, batch, stride, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.gen, self.batch = g, batch
        self.n_pages = batch * stride
        self.free = torch.randperm(self.n_pages, generator=g, device="cuda").int()
        self.table = torch.full((batch, stride), -1, dtype=torch.int32, device="cuda")
        self.cache = pa.cache_q4(PAT, self.n_pages, HKV, D)
        self.weights = [(1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16() for _ in range(2)]
        self.inv = (1e4 ** (-torch.arange(0, ROT, 2, device="cuda").double() / ROT)).float()
        self.held = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.ws = pa.decode_paged_q4_workspace(PAT, batch, HQ, HKV, D, stride * 64)

    def project(self, rows):
        return torch.randn((self.batch, rows, (HQ + 2 * HKV) * D), generator=self.gen, device="cuda").bfloat16()

    def attend(self, x, q_len):
        """the calls between the projection and the attention: (q, k, v), and the slots; nothing waits for the GPU"""
        rows = x.shape[1]
        q, k, v = (t.unflatten(2, (-1, D)).transpose(1, 2) for t in x.split([HQ * D, HKV * D, HKV * D], 2))
        slots, kv_len, taken = pa.page_tables(PAT, self.held, q_len, self.free, self.table, self.n_pages, rows)
        q, k = pa.qk_norm_rope(q, k, *self.weights, self.inv, q_start=self.held, q_len=q_len)
        pa.cache_store_q4(PAT, k, v, self.cache, slots)
        self.free.copy_(self.free[(torch.arange(self.n_pages, device="cuda") + taken) % self.n_pages])
        self.held.copy_(kv_len)
        return q, k, v

    def step(self, x, q_len, o, lse):
        q, k, v = self.attend(x, q_len)
        pa.decode_paged_q4(PAT, q[:, :, 0].contiguous(), self.cache, self.table, self.held, o=o, lse=lse, workspace=self.ws)
        return q, k, v


class Exact:
    """the rows that the cache stands for, kept in order"""

    def __init__(self, batch):
        self.k, self.v = ([np.zeros((HKV, 0, D)) for _ in range(batch)] for _ in range(2))

    def add(self, k, v, q_len):
        for i, n in enumerate(q_len):
            for rows, x in ((self.k, k), (self.v, v)):
                rows[i] = np.concatenate([rows[i], expand(*shrink(f64(x)[i, :, :n]))], 1)

    def check(self, q, o, lse):
        for i in range(len(self.k)):
            n = self.k[i].shape[1]
            if n == 0:
                assert (f64(o)[i] == 0).all() and (f64(lse)[i] == -np.inf).all()
                continue
            want, want_lse = orc.decode(f64(q)[i: i + 1, :, 0], self.k[i][None], self.v[i][None], [n], oracle_pattern(PAT))
            tol = 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -12 * np.abs(self.v[i]).max()
            assert (np.abs(f64(o)[i] - want[0]) <= tol).all()
            assert np.abs(f64(lse)[i] - want_lse[0]).max() <= 2.0 ** -13


def test_prompts_then_tokens_eager_and_replayed():
    lens, stride = [100, 0, 64, 333, 1], 8
    loop, exact = Loop(5, stride, 1), Exact(5)
    q, k, v = loop.attend(loop.project(333), i32(*lens))
    exact.add(k, v, lens)
    assert loop.held.tolist() == lens
    used = loop.table[loop.table >= 0].tolist()
    assert len(set(used)) == len(used) == sum(-(-n // 64) for n in lens)
    for b in (0, 3):                                       # the cache holds the prompt
        got = pa.cache_load_q4(PAT, loop.cache, loop.table, 333, length=i32(*lens))
        assert np.array_equal(f64(got[0])[b, :, : lens[b]], exact.k[b]) and np.array_equal(f64(got[1])[b, :, : lens[b]], exact.v[b])

    one = i32(1, 0, 1, 1, 1)                               # an idle place in the batch
    o, lse = torch.empty((5, HQ, D), dtype=torch.bfloat16, device="cuda"), torch.empty((5, HQ), device="cuda")
    for _ in range(2):
        q, k, v = loop.step(loop.project(1), one, o, lse)
        exact.add(k, v, one.tolist())
        exact.check(q, o, lse)

    x = loop.project(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                          # warm up on a copy of the state
        twin = Loop(5, stride, 1)
        twin.step(x, one, o.clone(), lse.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, k, v = loop.step(x, one, o, lse)
    for i in range(70):                                    # over the ends of pages
        x.copy_(loop.project(1))
        graph.replay()
        torch.cuda.synchronize()
        exact.add(k, v, one.tolist())
        if i % 10 == 9:
            exact.check(q, o, lse)
            pa.decode_paged_q4(PAT, q[:, :, 0].contiguous(), loop.cache, loop.table, loop.held, workspace=loop.ws)     # between replays
            torch.cuda.synchronize()
    assert loop.held.tolist() == [n + 72 * (j != 1) for j, n in enumerate(lens)]


def test_two_graphs_share_a_workspace_one_after_the_other():
    a, b = Loop(3, 4, 2), Loop(3, 4, 3)
    b.ws = a.ws
    graphs, states = [], []
    for loop in (a, b):
        x, one = loop.project(1), i32(1, 1, 1)
        o, lse = torch.empty((3, HQ, D), dtype=torch.bfloat16, device="cuda"), torch.empty((3, HQ), device="cuda")
        exact = Exact(3)
        q, k, v = loop.step(x, one, o, lse)
        exact.add(k, v, [1] * 3)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q, k, v = loop.step(x, one, o, lse)
        graphs.append(g)
        states.append((exact, q, k, v, o, lse, x, one))    # (the graph reads its inputs again at every replay)
    for _ in range(3):
        for g, (exact, q, k, v, o, lse, *_) in zip(graphs, states):
            g.replay()
            torch.cuda.synchronize()
            exact.add(k, v, [1] * 3)
            exact.check(q, o, lse)


def test_a_further_piece_against_the_loaded_cache():
    loop = Loop(1, 20, 4)
    loop.attend(loop.project(500), i32(500))
    q, k, v = loop.attend(loop.project(130), i32(130))
    kc, vc = pa.cache_load_q4(PAT, loop.cache, loop.table, 640, length=loop.held)
    cnt, idx, _ = pa.mask_build(PAT, 640)
    o, lse = pa.prefill_chunk(PAT, cnt, idx, q, kc, vc, 500)
    # its last row is the decode step's (which keeps 16 bits of P instead of 8)
    o1, lse1 = pa.decode_paged_q4(PAT, q[:, :, -1].contiguous(), loop.cache, loop.table, loop.held)
    want = f64(o1)
    assert (np.abs(f64(o)[:, :, -1] - want) <= 2.0 ** -7 * np.abs(want) + (2.0 ** -9 + 2.0 ** -11) * f64(vc.abs().max())).all()
    assert np.abs(f64(lse)[:, :, -1] - f64(lse1)).max() <= 2.0 ** -12


def test_on_another_stream():
    loop, exact = Loop(2, 10, 5), Exact(2)
    big = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            big = torch.tanh(big @ big)                    # the calls' inputs are made behind this
        x = loop.project(200) + 0 * big[0, 0].bfloat16()
        q, k, v = loop.attend(x, i32(200, 77))
        exact.add(k, v, [200, 77])
        o, lse = torch.empty((2, HQ, D), dtype=torch.bfloat16, device="cuda"), torch.empty((2, HQ), device="cuda")
        q, k, v = loop.step(loop.project(1), i32(1, 1), o, lse)
        exact.add(k, v, [1, 1])
    side.synchronize()
    exact.check(q, o, lse)
    by_handle = pa.decode_paged_q4(PAT, q[:, :, 0].contiguous(), loop.cache, loop.table, loop.held, stream=side)
    side.synchronize()
    assert torch.equal(by_handle[0], o) and torch.equal(by_handle[1], lse)


def test_two_calls_at_once():
    loops = [Loop(4, 10, 6), Loop(4, 10, 7)]
    streams = [torch.cuda.Stream() for _ in loops]
    exacts, out = [Exact(4) for _ in loops], []
    torch.cuda.synchronize()
    for loop, s in zip(loops, streams):
        with torch.cuda.stream(s):
            q, k, v = loop.attend(loop.project(300), i32(300, 5, 0, 150))
            o, lse = torch.empty((4, HQ, D), dtype=torch.bfloat16, device="cuda"), torch.empty((4, HQ), device="cuda")
            out.append((k, v, *loop.step(loop.project(1), i32(1, 1, 1, 1), o, lse), o, lse))
    torch.cuda.synchronize()
    for exact, (k0, v0, q, k, v, o, lse) in zip(exacts, out):
        exact.add(k0, v0, [300, 5, 0, 150])
        exact.add(k, v, [1] * 4)
        exact.check(q, o, lse)


def test_gradients_captured_in_a_graph():
    gen = torch.Generator("cuda").manual_seed(8)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, dq_out, dk_out = new(2, HQ, 150, D), new(2, HKV, 150, D), new(2, HQ, 150, D), new(2, HKV, 150, D)
    w, inv = (new(D), new(D)), (1e4 ** (-torch.arange(0, ROT, 2, device="cuda").double() / ROT)).float()
    ws = pa.qk_norm_rope_backward_workspace(2, HQ, HKV, 150, D)
    pa.qk_norm_rope_backward(q, k, *w, inv, dq_out, dk_out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pa.qk_norm_rope_backward(q, k, *w, inv, dq_out, dk_out, workspace=ws)
    for _ in range(4):
        for t in (q, k, dq_out, dk_out):
            t.copy_(new(*t.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = pa.qk_norm_rope_backward(q, k, *w, inv, dq_out, dk_out)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
