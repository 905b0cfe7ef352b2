"""What the binding's calls make themselves (outputs, workspaces) when a stream is given: on that stream, so that a fill or an earlier
use of the memory cannot come after the kernel.  Without a GPU: stand-ins for the streams and for the library."""
import ctypes
import inspect

import pytest
import torch

from paper_2503_03588_amd import binding as pa
from test_around_host import ordinary

PAT = pa.Pattern(64, 4, 1)
HERE = 0x10


class Streams:
    """torch.cuda's current stream, and what was made on which"""

    def __init__(self, monkeypatch):
        self.now, self.made, self.recorded = HERE, [], []
        me = self

        class Stream:
            def __init__(self, handle=None):
                self.cuda_stream = handle

        class Within:
            def __init__(self, s):
                self.s = s.cuda_stream

            def __enter__(self):
                self.before, me.now = me.now, self.s

            def __exit__(self, *e):
                me.now = self.before

        self.Stream = Stream
        for name, value in (("Stream", Stream), ("ExternalStream", Stream), ("stream", Within), ("current_stream", lambda device=None: Stream(me.now)),
                            ("default_stream", lambda device=None: Stream(0))):
            monkeypatch.setattr(torch.cuda, name, value)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: me.recorded.append(s.cuda_stream), raising=False)
        for name in ("empty", "zeros", "empty_like", "zeros_like"):
            monkeypatch.setattr(torch, name, self.noted(getattr(torch, name)))

    def noted(self, make):
        def f(*args, **kw):
            self.made.append(self.now)
            return make(*args, **{k: v for k, v in kw.items() if k != "device"})
        return f


def calls():
    q, q1 = torch.zeros(2, 4, 64, 64), torch.zeros(2, 4, 64)
    kv, one = torch.zeros(2, 2, 64, 64), torch.ones(2, dtype=torch.int32)
    cnt, idx, table = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 6, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32)
    lse = torch.zeros(2, 4, 64)
    yield pa.mask_build, (PAT, 128)
    yield pa.prefill, (PAT, cnt, idx, q, kv, kv)
    yield pa.prefill_chunk, (PAT, cnt, idx, q, kv, kv, 0)
    yield pa.prefill_chunk_paged, (PAT, cnt, idx, q, kv, kv, table, 0)
    yield pa.prefill_batch_paged, (PAT, cnt, idx, q, kv, kv, table, one, one)
    yield pa.prefill_varlen, (PAT, cnt, idx, q, kv, kv, one)
    yield pa.decode, (PAT, q1, kv, kv, one)
    yield pa.decode_paged, (PAT, q1, kv, kv, table, one)
    yield pa.backward, (PAT, cnt, idx, q, kv, kv, q, lse, q)
    made = {"page_tables": ("slots", "kv_len", "n_taken"), "qk_norm_rope": ("q_out", "k_out"),
            "qk_norm_rope_backward": ("dq", "dk", "dq_weight", "dk_weight", "workspace"), "cache_load_q4": ("k", "v"),
            "decode_paged_q4": ("o", "lse", "workspace")}
    for name, outs in made.items():
        f, args = getattr(pa, name), {k: v for k, v in ordinary()[name].items() if k not in outs}
        yield f, args
        if "q_len" in args and "inv_freq" in args:
            yield f, {**args, "q_len": None}


@pytest.fixture
def library(monkeypatch):
    class Entry:
        pass

    entry, real = Entry(), pa.lib()
    for name in pa.EXPORTS:
        f = getattr(real, name)
        plain = f.restype is ctypes.c_int and name not in ("powattn_version",)
        setattr(entry, name, (lambda *args: pa.OK) if plain else f)
    monkeypatch.setattr(pa, "lib", lambda: entry)
    monkeypatch.setattr(pa, "_on_this_gpu", lambda *tensors: None)
    monkeypatch.setattr(pa, "_native", None)


@pytest.mark.parametrize("how", ["a stream", "a handle", "the default stream's handle", "the current stream", "its handle"])
def test_what_a_call_makes_is_made_on_its_stream(library, monkeypatch, how):
    everything = list(calls())
    s = Streams(monkeypatch)
    stream, handle = {"a stream": (s.Stream(0x77), 0x77), "a handle": (0x77, 0x77), "the default stream's handle": (0, 0),
                      "the current stream": (s.Stream(HERE), HERE), "its handle": (HERE, HERE)}[how]
    for f, args in everything:
        s.made.clear()
        s.recorded.clear()
        f(*args, stream=stream) if isinstance(args, tuple) else f(**args, stream=stream)
        assert s.made and set(s.made) == {handle}, f.__name__
        assert s.recorded == ([] if handle == HERE else [HERE] * len(s.made)), f.__name__      # and used here as well
        assert s.now == HERE


def test_every_call_with_a_stream_is_looked_at():
    seen = {f.__name__ for f, _ in calls()} | {"decode_static", "cache_store_q4"}               # (these two make nothing)
    assert seen == {n for n, f in vars(pa).items() if inspect.isfunction(f) and not n.startswith("_") and "stream" in inspect.signature(f).parameters}
