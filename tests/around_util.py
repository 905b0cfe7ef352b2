"""64-bit definitions of what surrounds the attention calls: pages and slots, norm and rotation, the 4-bit format."""
import numpy as np
import torch

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def bf16(x):
    """float64 values of an array rounded to bf16 (to the nearest, ties to even)"""
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


# ---- pages and slots -----------------------------------------------------------------------------------------------------
def tables(block, q_start, q_len, q_rows, free, n_pages, table):
    """One token after the other: (table, slots, kv_len, number of pages taken)."""
    table = np.array(table)
    cap = table.shape[1] * block
    slots = np.full((len(q_start), q_rows), -1)
    kv_len, taken = [], 0
    for b in range(len(q_start)):
        s = min(max(int(q_start[b]), 0), cap)
        n = min(max(int(q_len[b]), 0), q_rows, cap - s)
        for r in range(n):
            blk, off = divmod(s + r, block)
            if off == 0:
                table[b, blk] = free[taken] if taken < len(free) else -1
                taken += 1
            if 0 <= table[b, blk] < n_pages:
                slots[b, r] = table[b, blk] * block + off
        kv_len.append(s + n)
    return table, slots, np.array(kv_len), taken


# ---- norm and rotation ---------------------------------------------------------------------------------------------------
def pairs(rot, interleaved):
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)


def norm_rope(x, w, inv_freq, start, eps, interleaved):
    """x [b,H,N,D] float64; returns (y, u): the result, and the rows before the rotation"""
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y = u.copy()
    if rot:
        pos = np.asarray(start, dtype=np.float64)[:, None] + np.arange(x.shape[2])
        a = (pos[..., None] * np.asarray(inv_freq, dtype=np.float64))[:, None]          # [b,1,N,rot/2]
        i, j = pairs(rot, interleaved)
        y[..., i] = u[..., i] * np.cos(a) - u[..., j] * np.sin(a)
        y[..., j] = u[..., i] * np.sin(a) + u[..., j] * np.cos(a)
    return y, u


def norm_rope_grad(x, w, inv_freq, start, eps, interleaved, dy, there):
    """there [b,N]: rows that exist.  Returns (dx, dw, parts) with parts the magnitudes of what dx and dw are sums of"""
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    du, mag = dy.copy(), np.abs(dy)
    if rot:
        pos = np.asarray(start, dtype=np.float64)[:, None] + np.arange(x.shape[2])
        a = (pos[..., None] * np.asarray(inv_freq, dtype=np.float64))[:, None]
        i, j = pairs(rot, interleaved)
        du[..., i] = dy[..., i] * np.cos(a) + dy[..., j] * np.sin(a)
        du[..., j] = dy[..., j] * np.cos(a) - dy[..., i] * np.sin(a)
        mag[..., i] = mag[..., j] = np.abs(dy[..., i]) + np.abs(dy[..., j])
    n = x * r
    dn = du * w
    dx = r * (dn - n * (dn * n).mean(-1, keepdims=True))
    keep = there[:, None, :, None]
    dw = np.where(keep, du * n, 0).sum((0, 1, 2))
    big_x = r * (mag * np.abs(w) + np.abs(n) * (mag * np.abs(w) * np.abs(n)).mean(-1, keepdims=True))
    return dx, dw, (big_x, np.where(keep, mag * np.abs(n), 0).sum((0, 1, 2)))


# ---- the 4-bit format ------------------------------------------------------------------------------------------------------
def shrink(x):
    """x [..., D] float64 -> (codes 0..15 [..., D], scale codes [..., D/32])"""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    m = np.abs(np.where(np.isfinite(g), g, 0)).max(-1)
    e = np.frexp(m)[1] - 1                                             # 2^e <= m < 2^(e+1)
    scale = np.where(m >= 1.75 * np.exp2(e.astype(float)), e - 1, e - 2)
    scale = np.clip(np.where(m == 0, -127, scale), -127, 125)
    y = np.where(bad[..., None], 0, g / np.exp2(scale.astype(float))[..., None])
    far = np.abs(np.abs(y)[..., None] - GRID)
    near = far.min(-1, keepdims=True)
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = even_first[(far[..., even_first] == near).argmax(-1)]
    code = np.where(np.signbit(y), code + 8, code)
    return code.reshape(x.shape), np.where(bad, 255, scale + 127)


def expand(code, scale):
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code % 8]
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(float) - 127))
    return (v.reshape(*code.shape[:-1], code.shape[-1] // 32, 32) * s[..., None]).reshape(code.shape)


def codes_of(rows):
    """[..., D/2] bytes -> [..., D] codes"""
    rows = rows.astype(np.int64)
    return np.stack([rows & 15, rows >> 4], -1).reshape(*rows.shape[:-1], -1)


def values_of(data, scales):
    """pages [n,H,B,D/2], scales [n,H,D/32,B] -> float64 [n,H,B,D]"""
    return expand(codes_of(data), scales.astype(np.int64).transpose(0, 1, 3, 2))

