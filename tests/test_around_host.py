"""What the calls around the attention refuse, on the host and before anything could be launched (no GPU needed): the C ABI's
statuses, and the binding's exceptions."""
import ctypes

import pytest
import torch

from paper_2503_03588_amd import binding as pa

FAKE = 0x10000          # a non-null "device pointer" that is never dereferenced on these paths
STRIDES = (ctypes.c_int64 * 3)(1 << 20, 128, 1024)


@pytest.fixture(scope="module")
def L():
    return pa.lib()


def _tables(L, pat=None, start=FAKE, n=2 * FAKE, batch=4, rows=10, free=3 * FAKE, n_free=9, n_pages=100, table=4 * FAKE, stride=16,
            slots=5 * FAKE, kv_len=6 * FAKE, taken=7 * FAKE):
    cp = (pat or pa.Pattern(64, 4, 1)).c()
    return L.powattn_page_tables(ctypes.byref(cp), start, n, batch, rows, free, n_free, n_pages, table, stride, slots, kv_len, taken,
                                 None)


def test_page_tables_argument_errors(L):
    for name in ("start", "n", "table", "slots", "kv_len", "taken", "free"):
        assert _tables(L, **{name: None}) == pa.INVALID_ARG, name
    for name in ("batch", "rows", "n_pages", "stride"):
        assert _tables(L, **{name: 0}) == pa.INVALID_ARG, name
    assert _tables(L, n_free=-1) == pa.INVALID_ARG
    for out in ("table", "slots", "kv_len", "taken"):                          # an output in the place of an input
        for where in (FAKE, 2 * FAKE, 3 * FAKE):
            assert _tables(L, **{out: where}) == pa.INVALID_ARG, out
    assert _tables(L, rows=16 * 64 + 1) == pa.INVALID_ARG
    assert _tables(L, pat=pa.Pattern(0, 4, 1)) == pa.INVALID_ARG
    assert _tables(L, n_pages=2 ** 31 // 64) == pa.UNSUPPORTED                  # slots are 32-bit numbers
    assert _tables(L, stride=2 ** 25) == pa.UNSUPPORTED
    assert L.powattn_page_tables(None, FAKE, 2 * FAKE, 4, 1, 3 * FAKE, 1, 1, 4 * FAKE, 1, 5 * FAKE, 6 * FAKE, 7 * FAKE, None) == pa.INVALID_ARG


def _rope(L, q=FAKE, qs=STRIDES, k=FAKE, ks=STRIDES, qw=FAKE, kw=FAKE, inv=FAKE, rot=128, flags=0, qo=FAKE, ko=FAKE, batch=2, hq=4, hkv=2,
          rows=100, d=128, dtype=pa.BF16, eps=1e-6):
    return L.powattn_qk_norm_rope(q, qs, k, ks, qw, kw, inv, rot, flags, None, None, qo, ko, batch, hq, hkv, rows, d, dtype, eps, None)


def _grad(L, q=FAKE, qs=STRIDES, k=FAKE, ks=STRIDES, qw=FAKE, kw=FAKE, inv=FAKE, rot=128, flags=0, gq=FAKE, gk=FAKE, dq=FAKE, dqs=STRIDES,
          dk=FAKE, dks=STRIDES, dqw=FAKE, dkw=FAKE, batch=2, hq=4, hkv=2, rows=100, d=128, dtype=pa.BF16, eps=1e-6, ws=FAKE, ws_bytes=None):
    if ws_bytes is None:
        ws_bytes = L.powattn_qk_norm_rope_backward_workspace_bytes(2, 4, 2, 100, 128)
    return L.powattn_qk_norm_rope_backward(q, qs, k, ks, qw, kw, inv, rot, flags, None, None, gq, gk, dq, dqs, dk, dks, dqw, dkw, batch, hq,
                                           hkv, rows, d, dtype, eps, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_rope, _grad])
def test_qk_norm_rope_argument_errors(L, call):
    names = ("q", "qs", "k", "ks", "qw", "kw", "inv") + (("qo", "ko") if call is _rope else ("gq", "gk", "dq", "dqs", "dk", "dks", "dqw", "dkw"))
    for name in names:
        assert call(L, **{name: None}) == pa.INVALID_ARG, name
    for name in ("batch", "hq", "hkv", "rows", "d"):
        assert call(L, **{name: 0}) == pa.INVALID_ARG, name
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(L, eps=eps) == pa.INVALID_ARG
    assert call(L, rot=-16) == pa.INVALID_ARG and call(L, rot=144) == pa.INVALID_ARG
    assert call(L, flags=2) == pa.INVALID_ARG
    assert call(L, rot=24) == pa.UNSUPPORTED
    assert call(L, d=96, rot=32) == pa.UNSUPPORTED
    assert call(L, dtype=5) == pa.UNSUPPORTED
    assert call(L, rows=2 ** 31) == pa.UNSUPPORTED


def test_qk_norm_rope_backward_workspace(L):
    assert _grad(L, ws=None) == pa.WORKSPACE_TOO_SMALL
    assert _grad(L, ws_bytes=100) == pa.WORKSPACE_TOO_SMALL
    assert _grad(L, ws=FAKE + 16) == pa.INVALID_ARG
    size = L.powattn_qk_norm_rope_backward_workspace_bytes
    assert size(0, 4, 2, 100, 128) == 0 and size(2, 4, 2, 100, 96) == 0
    assert 0 < size(1, 1, 1, 1, 64) < size(4, 32, 8, 32768, 128) < 4 << 20


def _store(L, pat=None, k=FAKE, ks=STRIDES, v=FAKE, vs=STRIDES, slots=FAKE, kp=FAKE, vp=FAKE, ksc=FAKE, vsc=FAKE, n_pages=100, batch=2, hkv=2,
           rows=10, d=128, dtype=pa.BF16):
    cp = (pat or pa.Pattern(64, 4, 1)).c()
    return L.powattn_cache_store_q4(ctypes.byref(cp), k, ks, v, vs, slots, kp, vp, ksc, vsc, n_pages, batch, hkv, rows, d, dtype, None)


def _load(L, pat=None, k=FAKE, v=FAKE, table=FAKE, stride=4, kp=FAKE, vp=FAKE, ksc=FAKE, vsc=FAKE, n_pages=100, batch=2, hkv=2, rows=10,
          d=128, dtype=pa.BF16):
    cp = (pat or pa.Pattern(64, 4, 1)).c()
    return L.powattn_cache_load_q4(ctypes.byref(cp), kp, vp, ksc, vsc, n_pages, table, stride, None, None, k, v, batch, hkv, rows, d, dtype,
                                   None)


@pytest.mark.parametrize("call", [_store, _load])
def test_cache_q4_argument_errors(L, call):
    for name in ("k", "v", "kp", "vp", "ksc", "vsc") + (("ks", "vs", "slots") if call is _store else ("table",)):
        assert call(L, **{name: None}) == pa.INVALID_ARG, name
    for name in ("batch", "hkv", "rows", "d", "n_pages") + (() if call is _store else ("stride",)):
        assert call(L, **{name: 0}) == pa.INVALID_ARG, name
    for name in ("kp", "vp", "ksc", "vsc"):
        assert call(L, **{name: FAKE + 8}) == pa.INVALID_ARG, name
    assert call(L, pat=pa.Pattern(64, -1, 1)) == pa.INVALID_ARG
    assert call(L, pat=pa.Pattern(48, 4, 1)) == pa.UNSUPPORTED
    assert call(L, pat=pa.Pattern(2048, 4, 1)) == pa.UNSUPPORTED
    assert call(L, d=96) == pa.UNSUPPORTED
    assert call(L, dtype=pa.F32) == pa.UNSUPPORTED
    assert call(L, n_pages=2 ** 31 // 64) == pa.UNSUPPORTED
    assert call(L, batch=2 ** 20, rows=2 ** 12) == pa.UNSUPPORTED


def _decode(L, pat=None, q=FAKE, kp=FAKE, vp=FAKE, ksc=FAKE, vsc=FAKE, n_pages=100, table=FAKE, stride=16, kv_len=FAKE, o=FAKE, batch=2, hq=8,
            hkv=2, d=128, dtype=pa.BF16, scale=0.0, ws=FAKE, ws_bytes=1 << 24):
    cp = (pat or pa.Pattern(64, 4, 1)).c()
    return L.powattn_decode_paged_q4(ctypes.byref(cp), q, kp, vp, ksc, vsc, n_pages, table, stride, kv_len, o, None, batch, hq, hkv, d, dtype,
                                     scale, ws, ws_bytes, None)


def test_decode_paged_q4_argument_errors(L):
    for name in ("q", "kp", "vp", "ksc", "vsc", "table", "kv_len", "o"):
        assert _decode(L, **{name: None}) == pa.INVALID_ARG, name
    for name in ("batch", "hq", "hkv", "d", "n_pages", "stride"):
        assert _decode(L, **{name: 0}) == pa.INVALID_ARG, name
    assert _decode(L, hq=7) == pa.INVALID_ARG
    assert _decode(L, scale=float("nan")) == pa.INVALID_ARG
    for name in ("q", "kp", "vp", "ksc", "vsc"):
        assert _decode(L, **{name: FAKE + 8}) == pa.INVALID_ARG, name
    assert _decode(L, d=96) == pa.UNSUPPORTED
    assert _decode(L, dtype=pa.F32) == pa.UNSUPPORTED
    assert _decode(L, pat=pa.Pattern(48, 4, 1)) == pa.UNSUPPORTED
    assert _decode(L, pat=pa.Pattern(64, 1, 0, pa.DENSE)) == pa.UNSUPPORTED
    assert _decode(L, hq=34) == pa.UNSUPPORTED                                   # 17 heads on one
    assert _decode(L, n_pages=2 ** 31 // 64) == pa.UNSUPPORTED
    assert _decode(L, batch=70000, ws_bytes=1 << 40) == pa.UNSUPPORTED
    assert _decode(L, ws=None) == pa.WORKSPACE_TOO_SMALL
    assert _decode(L, ws_bytes=0) == pa.WORKSPACE_TOO_SMALL
    assert _decode(L, ws=FAKE + 64) == pa.INVALID_ARG
    cp = pa.Pattern(64, 4, 1).c()
    size = L.powattn_decode_paged_q4_workspace_bytes
    assert size(None, 2, 8, 2, 128, 1024) == 0 and size(ctypes.byref(cp), 2, 7, 2, 128, 1024) == 0
    assert size(ctypes.byref(cp), 2, 8, 2, 128, 0) == 0 and size(ctypes.byref(cp), 2, 8, 2, 128, 1024) > 0


# ---- the binding -----------------------------------------------------------------------------------------------------------
PAT = pa.Pattern(64, 4, 1)
B, HQ, HKV, N, D = 2, 4, 2, 10, 64


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def ordinary():
    cache = (u8(5, HKV, 64, 32), u8(5, HKV, 64, 32), u8(5, HKV, 2, 64), u8(5, HKV, 2, 64))
    rope = dict(q=bf16(B, HQ, N, D), k=bf16(B, HKV, N, D), q_weight=bf16(D), k_weight=bf16(D), inv_freq=torch.zeros(16), q_start=i32(B),
                q_len=i32(B))
    return {
        "page_tables": dict(pattern=PAT, q_start=i32(B), q_len=i32(B), free_pages=i32(7), block_table=i32(B, 3), n_pages=9, q_rows=N,
                            slots=i32(B, N), kv_len=i32(B), n_taken=i32(1)),
        "qk_norm_rope": dict(**rope, q_out=bf16(B, HQ, N, D), k_out=bf16(B, HKV, N, D)),
        "qk_norm_rope_backward": dict(**rope, dq_out=bf16(B, HQ, N, D), dk_out=bf16(B, HKV, N, D), dq=bf16(B, HQ, N, D),
                                      dk=bf16(B, HKV, N, D), dq_weight=torch.zeros(D), dk_weight=torch.zeros(D), workspace=u8(1 << 16)),
        "cache_store_q4": dict(pattern=PAT, k=bf16(B, HKV, N, D), v=bf16(B, HKV, N, D), cache=cache, slots=i32(B, N)),
        "cache_load_q4": dict(pattern=PAT, cache=cache, block_table=i32(B, 3), rows=N, start=i32(B), length=i32(B), k=bf16(B, HKV, N, D),
                              v=bf16(B, HKV, N, D)),
        "decode_paged_q4": dict(pattern=PAT, q=bf16(B, HQ, D), cache=cache, block_table=i32(B, 3), kv_len=i32(B), o=bf16(B, HQ, D),
                                lse=torch.zeros(B, HQ), workspace=u8(1 << 16)),
    }


class Entry:
    """Stands in for the library: what reaches it is written down."""

    def __init__(self):
        self.seen = []
        real = pa.lib()
        for name in pa.EXPORTS:
            f = getattr(real, name)
            setattr(self, name, self._called(name) if name[8:] in ordinary() else f)

    def _called(self, name):
        def f(*args):
            self.seen.append(name)
            return pa.OK
        return f


@pytest.fixture
def entry(monkeypatch):
    e = Entry()
    monkeypatch.setattr(pa, "lib", lambda: e)
    monkeypatch.setattr(pa, "_stream", lambda stream=None: 0)
    monkeypatch.setattr(pa, "_on_this_gpu", lambda *tensors: None)
    monkeypatch.setattr(pa, "_native", None)
    return e


@pytest.mark.parametrize("name", sorted(ordinary()))
def test_tensors_that_are_not_what_a_call_takes(entry, name):
    args = ordinary()[name]
    getattr(pa, name)(**args)
    assert entry.seen == ["powattn_" + name]
    strided = {"q", "k", "v", "dq", "dk"} if name != "decode_paged_q4" else set()
    optional = {"q_start", "q_len"} if "inv_freq" in args else {"start", "length"}
    changed = {a: t for a, t in args.items() if isinstance(t, torch.Tensor) and a != "workspace"}
    changed.update({("cache", i): t for i, t in enumerate(args.get("cache", ()))})
    for a, t in changed.items():
        def refused(new, what):
            entry.seen.clear()
            call = dict(args)
            if isinstance(a, tuple):
                call["cache"] = tuple(new if i == a[1] else x for i, x in enumerate(args["cache"]))
            else:
                call[a] = new
            with pytest.raises((ValueError, pa.PowattnError, IndexError)):
                getattr(pa, name)(**call)
            assert not entry.seen, (a, what)

        refused(t.to(torch.float16), "another type")
        refused(t[None], "a dimension more")
        if a not in ("inv_freq", "free_pages", "block_table"):
            wide = torch.cat([t, t], -1)
            refused(wide, "a longer last dimension")
        wide = torch.stack([t, t], -1)[..., 0]
        if wide.numel() > 1:
            refused(wide, "components that are apart")
        if t.dim() > 1 and not (a in strided and name != "cache_load_q4"):
            refused(torch.cat([t, t], 1).narrow(1, 0, t.shape[1]), "rows that are apart")
        if a in optional:
            entry.seen.clear()
            getattr(pa, name)(**{**args, a: None})
            assert entry.seen


def test_gradients_into_rows_that_overlap(entry):
    args = ordinary()["qk_norm_rope_backward"]
    one = bf16(1, HQ, N, D)
    with pytest.raises(ValueError, match="overlap"):
        pa.qk_norm_rope_backward(**{**args, "dq": one.expand(B, -1, -1, -1)})
    with pytest.raises(ValueError, match="overlap"):
        pa.qk_norm_rope_backward(**{**args, "dk": bf16(B * N * HKV * D).as_strided((B, HKV, N, D), (N * D, D, D // 2, 1))})
    assert not entry.seen
    whole = bf16(B, N, (HQ + 2 * HKV) * D)                 # side by side in the gradient of the projections' output
    dq = whole[..., : HQ * D].unflatten(2, (-1, D)).transpose(1, 2)
    dk = whole[..., HQ * D: (HQ + HKV) * D].unflatten(2, (-1, D)).transpose(1, 2)
    pa.qk_norm_rope_backward(**{**args, "dq": dq, "dk": dk})
    assert entry.seen


def test_workspaces_that_are_too_small():
    for size in (pa.qk_norm_rope_backward_workspace, pa.decode_paged_q4_workspace):
        with pytest.raises(pa.PowattnError):
            size(*((PAT,) if size is pa.decode_paged_q4_workspace else ()), 0, HQ, HKV, 100, 128, device="cpu")


@pytest.mark.parametrize("name", sorted(ordinary()))
def test_tensors_in_ordinary_memory(monkeypatch, name):
    monkeypatch.setattr(pa, "_native", None)
    with pytest.raises(ValueError, match="current GPU"):
        getattr(pa, name)(**ordinary()[name])


def test_a_status_is_raised(entry):
    entry.powattn_page_tables = lambda *args: pa.UNSUPPORTED
    with pytest.raises(pa.PowattnError, match="powattn_page_tables: status 2"):
        pa.page_tables(**ordinary()["page_tables"])
