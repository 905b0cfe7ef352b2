"""The calls around the attention go to the library through Python or through csrc/host.cpp: each call, ordinary and then altered
in one place at a time, goes both ways over a stand-in for the library, and has to reach it with the same arguments, or not
at all and with the same exception."""
import ctypes

import pytest
import torch

from host_on_cpu import STREAM, host_cpu  # noqa: F401 (fixture)
from paper_2503_03588_amd import binding as pa
from test_around_host import D, HKV, HQ, N, B, bf16, i32, ordinary, u8

NEW = {"page_tables": ("slots", "kv_len", "n_taken"), "qk_norm_rope": ("q_out", "k_out"), "qk_norm_rope_backward": ("dq_weight", "dk_weight"),
       "cache_store_q4": (), "cache_load_q4": ("k", "v"), "decode_paged_q4": ("o", "lse")}       # outputs that a call makes itself
ORDER = {
    "page_tables": "q_start q_len free_pages block_table n_pages q_rows slots kv_len n_taken",
    "qk_norm_rope": "q k q_weight k_weight inv_freq q_start q_len eps interleaved q_out k_out",
    "qk_norm_rope_backward": "q k q_weight k_weight inv_freq q_start q_len eps interleaved dq_out dk_out dq dk dq_weight dk_weight workspace",
    "cache_store_q4": "k v cache slots",
    "cache_load_q4": "cache block_table rows start length k v",
    "decode_paged_q4": "q cache block_table kv_len o lse softmax_scale workspace want_lse",
}
DEFAULTS = {"eps": 1e-6, "interleaved": False, "softmax_scale": 0.0, "want_lse": True}


class StandIn:
    def __init__(self):
        self.seen, self.answers, real = [], [], pa.lib()
        for name in pa.EXPORTS:
            f = getattr(real, name)
            mine = name[8:] in ORDER
            setattr(self, name, ctypes.CFUNCTYPE(ctypes.c_int, *f.argtypes)(self._called(name)) if mine else f)

    def _called(self, name):
        def f(*args):
            plain = []
            for x in args:
                if isinstance(x, ctypes.POINTER(ctypes.c_int64)):
                    x = tuple(x[:3])
                elif isinstance(x, ctypes.POINTER(pa._CPattern)):
                    x = tuple(getattr(x.contents, n) for n, _ in pa._CPattern._fields_)
                plain.append("nan" if x != x else x)
            self.seen.append((name, plain))
            return self.answers.pop(0) if self.answers else pa.OK
        return f


@pytest.fixture
def stand_in(host_cpu, monkeypatch):  # noqa: F811
    fake = StandIn()
    host_cpu.bind(*(ctypes.cast(getattr(fake, "powattn_" + n), ctypes.c_void_p).value for n in pa._NATIVE_ENTRY_POINTS),
                  torch.Tensor, lambda: 0, lambda device: STREAM, pa._check)
    monkeypatch.setattr(pa, "lib", lambda: fake)
    monkeypatch.setattr(pa, "_stream", lambda stream=None: STREAM)
    monkeypatch.setattr(pa, "_on_this_gpu", lambda *tensors: None)
    monkeypatch.setattr(pa, "_native", host_cpu)
    return fake


class Sub(torch.Tensor):
    pass


def alterations(t):
    yield "fp32", t.float()
    yield "bf16", t.bfloat16()
    yield "int64", t.long()
    yield "bytes", t.to(torch.uint8)
    yield "a dimension less", t[0].contiguous()
    yield "a dimension more", t[None]
    for dim in range(t.dim()):
        yield f"dimension {dim} longer", torch.cat([t, t], dim)
        if t.shape[dim] > 1:
            yield f"dimension {dim} shorter", t.narrow(dim, 0, t.shape[dim] - 1).contiguous()
            yield f"dimension {dim} not contiguous", torch.cat([t, t], dim).narrow(dim, 0, t.shape[dim])
            yield f"dimension {dim} reversed in memory", t.transpose(0, dim).contiguous().transpose(0, dim)
            yield f"dimension {dim} expanded", t.narrow(dim, 0, 1).expand(t.shape)
    yield "empty", t[:0]
    yield "a subclass", t.as_subclass(Sub)
    yield "a parameter", torch.nn.Parameter(t, requires_grad=t.is_floating_point())
    yield "a negated view", torch._neg_view(t)
    yield "none", None
    yield "an array", t.float().numpy()


def cases(name):
    args = ordinary()[name]
    yield "as it is", args
    yield "outputs made by the call", {k: v for k, v in args.items() if k not in NEW[name]}
    if "workspace" in args:
        for ws in (None, args["workspace"][:8], args["workspace"].view(torch.int32), args["workspace"][::2]):
            yield f"workspace {ws if ws is None else tuple(ws.shape)}", {**args, "workspace": ws}
    if name == "qk_norm_rope_backward":
        yield "gradients made by the call", {k: v for k, v in args.items() if k not in ("dq", "dk")}
        whole = bf16(B, N, (HQ + 2 * HKV) * D)
        parts = [x.unflatten(2, (-1, D)).transpose(1, 2) for x in whole.split([HQ * D, HKV * D, HKV * D], 2)]
        yield "views of one gradient", {**args, "dq": parts[0], "dk": parts[1]}
    if "eps" in DEFAULTS and "q_weight" in args:
        for eps in (0, 0.0, 1, -1.0, float("nan"), "x", None):
            yield f"eps {eps!r}", {**args, "eps": eps}
        for inter in (True, False, 1, 0, None):
            yield f"interleaved {inter!r}", {**args, "interleaved": inter}
    if name == "decode_paged_q4":
        for scale in (0.25, 0, -1.0, float("nan"), 1e300, None):
            yield f"scale {scale!r}", {**args, "softmax_scale": scale}
        for lse in (torch.zeros(B, HQ), None):
            for want in (True, False, 1, 0, None):
                yield f"lse {lse is not None}, want_lse {want!r}", {**args, "lse": lse, "want_lse": want}
    if "pattern" in args:
        for pat in (pa.Pattern(128, 3, 1), pa.Pattern(64, 3, 1, pa.DENSE), pa.Pattern(-1, 3, 1)):
            yield repr(pat), {**args, "pattern": pat}
    for n in ("n_pages", "q_rows", "rows"):
        if n in args:
            for x in (0, 1, -1, 2 ** 40, True, 3.0, None):
                yield f"{n} {x!r}", {**args, n: x}
    if "cache" in args:
        yield "a cache of three", {**args, "cache": args["cache"][:3]}
        yield "a list", {**args, "cache": list(args["cache"])}
        yield "a CacheQ4", {**args, "cache": pa.CacheQ4(*args["cache"])}
        yield "a cache of other heads", {**args, "cache": (u8(5, 3, 64, 32), u8(5, 3, 64, 32), u8(5, 3, 2, 64), u8(5, 3, 2, 64))}
        for i, t in enumerate(args["cache"]):
            for how, changed in alterations(t):
                yield f"cache[{i}]: {how}", {**args, "cache": tuple(changed if j == i else x for j, x in enumerate(args["cache"]))}
    for arg, t in args.items():
        if isinstance(t, torch.Tensor):
            for how, changed in alterations(t):
                yield f"{arg}: {how}", {**args, arg: changed}


def outcome(fake, name, args):
    fake.seen.clear()
    try:
        result = getattr(pa, name)(**args)
    except Exception as e:
        assert not fake.seen
        return type(e).__name__
    (entry, passed), = fake.seen
    assert entry == "powattn_" + name
    result = () if result is None else result
    known = {t.data_ptr() for v in args.values() for t in (v if isinstance(v, (tuple, list)) else (v,)) if isinstance(t, torch.Tensor)}
    mine = {t.data_ptr() for t in result if isinstance(t, torch.Tensor)} - known
    if "workspace" in ORDER[name] and args.get("workspace") is None:
        mine.add(passed[-3])
    return tuple("new" if x in mine else x for x in passed), [(tuple(t.shape), t.dtype, t.stride()) if isinstance(t, torch.Tensor) else t for t in result]


@pytest.mark.parametrize("name", sorted(ORDER))
def test_both_ways_call_the_library_alike(stand_in, monkeypatch, name):
    host, calls, natively = pa._native, 0, 0
    for what, args in cases(name):
        monkeypatch.setattr(pa, "_native", host)
        with_native = outcome(stand_in, name, args)
        monkeypatch.setattr(pa, "_native", None)
        assert with_native == outcome(stand_in, name, args), what
        calls += 1
        if what in ("as it is", "outputs made by the call", "views of one gradient", "a CacheQ4"):
            values = [args.get(k, DEFAULTS.get(k)) for k in ORDER[name].split()]
            first = (args["pattern"]._values,) if "pattern" in args else ()
            assert getattr(host, name)(*first, *values) is not NotImplemented, what              # (these do go the native way)
            natively += 1
    assert calls > 60 and natively >= 2


@pytest.mark.parametrize("name", sorted(ORDER))
def test_a_status_is_raised_once(stand_in, name):
    stand_in.answers = [pa.HIP_ERROR]
    with pytest.raises(pa.PowattnError, match=f"powattn_{name}: status 4"):
        getattr(pa, name)(**ordinary()[name])
    assert len(stand_in.seen) == 1


def test_zeros_where_rows_may_be_left_out(stand_in):
    args = {k: v for k, v in ordinary()["qk_norm_rope"].items() if k not in ("q_out", "k_out")}
    for t in pa.qk_norm_rope(**args):
        assert not t.any()
    args = {k: v for k, v in ordinary()["cache_load_q4"].items() if k not in ("k", "v")}
    for t in pa.cache_load_q4(**args):
        assert not t.any()


def test_the_rows_of_a_fused_projection(stand_in):
    whole = bf16(B, N, (HQ + 2 * HKV) * D)
    q, k, v = (x.unflatten(2, (-1, D)).transpose(1, 2) for x in whole.split([HQ * D, HKV * D, HKV * D], 2))
    args = ordinary()["qk_norm_rope"]
    pa.qk_norm_rope(**{**args, "q": q, "k": k})
    passed = stand_in.seen[-1][1]
    wide = (HQ + 2 * HKV) * D
    assert passed[0] == whole.data_ptr() and passed[2] == whole.data_ptr() + 2 * HQ * D
    assert passed[1] == passed[3] == (N * wide, D, wide)
    pa.cache_store_q4(**{**ordinary()["cache_store_q4"], "v": v, "slots": i32(B, N)})
    assert stand_in.seen[-1][1][4] == (N * wide, D, wide)
