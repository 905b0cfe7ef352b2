"""Outputs of the calls around the attention that share memory with inputs or with one another are refused, on the host and before
anything could be launched (no GPU needed; the addresses are never dereferenced)."""
import ctypes

import pytest

from paper_2503_03588_amd import binding as pa

B, HQ, HKV, N, D = 2, 4, 2, 100, 128
MIB = 1 << 20


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def contiguous(heads):
    return strides(heads * N * D, N * D, D)


WIDE = (HQ + 2 * HKV) * D
FUSED = strides(N * WIDE, D, WIDE)                         # rows of a projection's output


def forward(q=(MIB, FUSED), k=(MIB + 2 * HQ * D, FUSED), q_out=2 * MIB, k_out=3 * MIB):
    return pa.lib().powattn_qk_norm_rope(q[0], q[1], k[0], k[1], 64, 64, 64, D, 0, None, None, q_out, k_out, B, HQ, HKV, N, D, pa.BF16, 1e-6,
                                         None)


def gradients(q=(MIB, FUSED), k=(MIB + 2 * HQ * D, FUSED), dq_out=2 * MIB, dk_out=3 * MIB, dq=(4 * MIB, FUSED), dk=(4 * MIB + 2 * HQ * D, FUSED),
              dq_weight=5 * MIB, dk_weight=6 * MIB):
    return pa.lib().powattn_qk_norm_rope_backward(q[0], q[1], k[0], k[1], 64, 64, 64, D, 0, None, None, dq_out, dk_out, dq[0], dq[1], dk[0],
                                                  dk[1], dq_weight, dk_weight, B, HQ, HKV, N, D, pa.BF16, 1e-6, 8 * MIB, 4 * MIB, None)


@pytest.mark.parametrize("how", [
    dict(dk=(4 * MIB, FUSED)),                             # one view for both
    dict(dk=(4 * MIB + 2 * (HQ - 1) * D, FUSED)),          # ... beginning in the other's last head
    dict(dk=(4 * MIB + 2 * HQ * D - 2, FUSED)),            # ... or its last component
    dict(dq=(4 * MIB, contiguous(HQ)), dk=(4 * MIB + 2 * B * HQ * N * D - 2, contiguous(HKV))),
    dict(dq=(MIB, FUSED), dk=(MIB + 2 * HQ * D, FUSED)),   # in the place of the inputs
    dict(dk=(MIB, FUSED)),
    dict(dq=(MIB + 2 * HQ * D, FUSED)),
    dict(dq=(2 * MIB, contiguous(HQ))),                    # ... of the upstream gradients
    dict(dk=(2 * MIB, contiguous(HKV))),
    dict(dk=(3 * MIB + 2 * N * D, contiguous(HKV))),
    dict(dq=(3 * MIB, FUSED)),
    dict(dk_weight=5 * MIB),
    dict(dk_weight=5 * MIB + 4 * D - 4),
])
def test_gradients_that_share_memory(how):
    assert gradients(**how) == pa.INVALID_ARG


@pytest.mark.parametrize("how", [
    dict(k_out=2 * MIB),
    dict(k_out=2 * MIB + 2 * B * HQ * N * D - 2),
    dict(q_out=MIB),
    dict(k_out=MIB + 2 * B * N * WIDE - 2 * 3 * HKV * D),
    dict(q=(2 * MIB, contiguous(HQ))),
    dict(k=(2 * MIB, contiguous(HKV))),
    dict(k=(3 * MIB, contiguous(HKV))),
])
def test_rows_that_share_memory(how):
    assert forward(**how) == pa.INVALID_ARG


def tables(start=MIB, n=2 * MIB, free=3 * MIB, table=4 * MIB, slots=5 * MIB, kv_len=6 * MIB, taken=7 * MIB):
    cp = pa.Pattern(64, 4, 1).c()
    return pa.lib().powattn_page_tables(ctypes.byref(cp), start, n, 40, 10, free, 9, 100, table, 16, slots, kv_len, taken, None)


@pytest.mark.parametrize("how", [
    dict(kv_len=MIB + 4),                                  # the lengths of all sequences but the first
    dict(kv_len=MIB - 4 * 39),
    dict(kv_len=2 * MIB + 4 * 39),
    dict(taken=MIB + 4 * 39),
    dict(taken=3 * MIB + 4 * 8),
    dict(slots=2 * MIB - 4 * 399),
    dict(table=3 * MIB - 4 * 639),
    dict(table=3 * MIB + 4),
    dict(kv_len=7 * MIB),                                  # one output in another
    dict(taken=5 * MIB + 4 * 399),
    dict(slots=4 * MIB + 4 * 639),
    dict(kv_len=4 * MIB + 4),
])
def test_page_tables_that_share_memory(how):
    assert tables(**how) == pa.INVALID_ARG


PAGES, ROWS = 16 * 2 * 64 * 64, 2 * B * HKV * N * D        # bytes of 16 pages of two heads, and of rows that are loaded


def store(kp=MIB, vp=2 * MIB, ks=3 * MIB, vs=4 * MIB):
    cp = pa.Pattern(64, 4, 1).c()
    return pa.lib().powattn_cache_store_q4(ctypes.byref(cp), 5 * MIB, contiguous(HKV), 6 * MIB, contiguous(HKV), 64, kp, vp, ks, vs, 16, B, HKV,
                                           N, D, pa.BF16, None)


def load(kp=MIB, vp=2 * MIB, ks=3 * MIB, vs=4 * MIB, k=5 * MIB, v=6 * MIB):
    cp = pa.Pattern(64, 4, 1).c()
    return pa.lib().powattn_cache_load_q4(ctypes.byref(cp), kp, vp, ks, vs, 16, 64, 4, None, None, k, v, B, HKV, N, D, pa.BF16, None)


@pytest.mark.parametrize("how", [dict(vp=MIB), dict(vp=MIB + PAGES - 16), dict(vs=3 * MIB), dict(ks=4 * MIB + PAGES // 16 - 16), dict(ks=2 * MIB + 16)])
def test_a_cache_that_shares_memory(how):
    assert store(**how) == pa.INVALID_ARG


@pytest.mark.parametrize("how", [dict(v=5 * MIB), dict(v=5 * MIB + ROWS - 16), dict(k=MIB), dict(v=2 * MIB + PAGES - 16), dict(k=3 * MIB)])
def test_loaded_rows_that_share_memory(how):
    assert load(**how) == pa.INVALID_ARG
