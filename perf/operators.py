"""The operators around the attention calls, as cases that can be timed: page tables and slot maps, the norm of queries and
keys with the rotation (and its gradients), the cache of 4-bit floats, and the decode step over it.

`run()` makes the library's calls where `own` is true; elsewhere it computes the same in elementary torch operations.

A case's "kind":
  tables     powattn_page_tables: pages and slots of a serving step's new tokens
  rope       powattn_qk_norm_rope
  rope_grad  powattn_qk_norm_rope_backward
  store      powattn_cache_store_q4, and powattn_cache_load_q4 of the rows just stored
  decode     powattn_decode_paged_q4
  step       one decode step of a layer: tables, norm and rotation, store, decode
"""
import math

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _case(kind, name=None, **kw):
    c = {"kind": kind, "dtype": "bf16", "batch": 1, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "block": 64, "window": 4, "sink": 1, "rows": 1, "len_lo": 0, "len_hi": 0, "ragged": False, "idle": 0}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One new token for every sequence of a serving batch: a page every 64th time.  Latency counts.
        _case("tables", "tables_step", batch=128, len_lo=1000, len_hi=16383),
        # A serving step's prefill work: pieces of many prompts, with different contexts so far.
        _case("tables", "tables_prompts", batch=32, rows=2048, len_lo=0, len_hi=61000, ragged=True),
        # Full precision, a partial rotation in neighbouring pairs, a short padded batch: what a research model runs.
        _case("rope", "rope_f32_1k", dtype="f32", batch=2, hq=4, hkv=2, d=64, rot=32, rows=1000, interleaved=True, ragged=True),
        # The queries and keys of one layer over an ordinary long prompt, out of a fused projection.
        _case("rope", "rope_32k", hq=28, hkv=4, rows=32768),
        # Gradients, full precision, odd length.
        _case("rope_grad", "grad_f32_777", dtype="f32", batch=2, hq=8, hkv=2, d=64, rot=64, rows=777, ragged=True),
        # Gradients of one layer in training on long sequences; the largest pass.
        _case("rope_grad", "grad_32k", hq=28, hkv=4, rows=32768),
        # The rows of one decode step of a serving batch into the cache.
        _case("store", "store_step", batch=128, len_lo=1000, len_hi=16383),
        # The rows of a step's prompt pieces into the cache, and out again for the next pieces.
        _case("store", "store_prompts", batch=32, rows=2048, len_lo=0, len_hi=4096, ragged=True),
        # Generation for one user: the smallest attention call there is.
        _case("decode", "decode_b1", len_lo=32001, len_hi=32001),
        # Generation for a small batch with long contexts.
        _case("decode", "decode_b16_64k", batch=16, len_lo=65536, len_hi=65536),
        # Generation for a large serving batch of mixed contexts.
        _case("decode", "decode_b128", batch=128, len_lo=1000, len_hi=16384),
        # One layer's whole decode step, two places of the padded batch idle.
        _case("step", "step_b64", batch=64, len_lo=500, len_hi=20000, idle=2),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("tables", "rope", "rope_grad", "store", "decode", "step"))
    d = rng.choice((64, 128))
    hkv = rng.choice((1, 2, 3, 4, 8))
    c = dict(d=d, hkv=hkv, hq=hkv * rng.choice((1, 2, 4, 5, 7, 8)), rot=rng.choice((d, d, d // 2, 16)),
             interleaved=rng.random() < 0.3, block=rng.choice((64, 64, 128, 256)), window=rng.randint(1, 6), sink=rng.randint(0, 2))
    if kind in ("rope", "rope_grad"):
        c["dtype"] = rng.choice(("bf16", "bf16", "f32"))
        c["batch"] = _log(rng, 1, 16)
        most = 32768 * 32 * 128 * 2 // (c["batch"] * (c["hq"] + hkv) * d * (4 if c["dtype"] == "f32" else 2))
        c["rows"] = _log(rng, 1, min(32768, most))
        c["ragged"] = c["rows"] > 1 and rng.random() < 0.5
        c["len_hi"] = _log(rng, 1, 1000000)
        c["len_lo"] = rng.randint(0, c["len_hi"])
    elif kind in ("tables", "store"):
        c["batch"] = _log(rng, 1, 256 if kind == "tables" else 64)
        c["rows"] = _log(rng, 1, max(1, min(2048, 65536 // c["batch"])))
        c["ragged"] = c["rows"] > 1
        c["len_hi"] = _log(rng, 1, 60000 if kind == "tables" else 4096)
        c["len_lo"] = rng.randint(0, c["len_hi"])
    else:
        c["batch"] = _log(rng, 1, 128)
        c["len_hi"] = _log(rng, 2, max(2, min(131072, 2097152 // c["batch"])))
        c["len_lo"] = rng.randint(1, c["len_hi"])
        c["idle"] = rng.choice((0, 0, 1)) if c["batch"] > 1 else 0
    return _case(kind, **c)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _lengths(c, gen, dev):
    """q_start and q_len of a step's sequences; the idle places of the batch come first."""
    b = c["batch"]
    start = torch.randint(c["len_lo"], c["len_hi"] + 1, (b,), generator=gen, device=dev, dtype=torch.int32)
    n = torch.full((b,), c["rows"], device=dev, dtype=torch.int32)
    if c["ragged"]:
        n = torch.randint(0, c["rows"] + 1, (b,), generator=gen, device=dev, dtype=torch.int32)
        n[0] = c["rows"]
    start[: c["idle"]] = 0
    n[: c["idle"]] = 0
    return start, n


def _stride(c, extra):
    return -(-(c["len_hi"] + extra) // c["block"])


def _pages(c, gen, dev, held, extra):
    """A shuffled pool: the table of the pages that the sequences hold, and the list of the free ones."""
    b, stride = c["batch"], _stride(c, extra)
    n_pages = b * stride + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    blocks = (held.long() + c["block"] - 1) // c["block"]
    table = order[: b * stride].view(b, stride).clone()
    mine = torch.arange(stride, device=dev)[None] < blocks[:, None]
    free = torch.cat([table[~mine], order[b * stride:]])
    return torch.where(mine, table, -1).to(torch.int32), free.contiguous(), n_pages


def _fused(c, gen, dev, heads, dtype):
    """Queries, keys and values (as many as `heads` says) as views of one projection's output [batch, rows, heads * d]."""
    d = c["d"]
    x = torch.randn((c["batch"], c["rows"], sum(heads) * d), generator=gen, device=dev, dtype=torch.float32).to(dtype)
    return [t.unflatten(2, (-1, d)).transpose(1, 2) for t in x.split([h * d for h in heads], dim=2)]


def _rope_inputs(c, gen, dev):
    t = TYPES[c["dtype"]]
    weights = [(1 + 0.2 * torch.randn(c["d"], generator=gen, device=dev)).to(t) for _ in range(2)]
    inv_freq = 1000000.0 ** (-torch.arange(0, c["rot"], 2, device=dev, dtype=torch.float64) / c["rot"])
    return {"q_weight": weights[0], "k_weight": weights[1], "inv_freq": inv_freq.float()}


def _filled_cache(c, gen, dev, n_pages):
    """Pages of keys and values of which some components are larger than others, as trained keys are."""
    d, hkv, B = c["d"], c["hkv"], c["block"]
    gain = 1 + 2 * torch.rand((hkv, 1, d), generator=gen, device=dev)
    shapes = {"k": (n_pages, hkv, B, d // 2), "ks": (n_pages, hkv, d // 32, B)}
    cache = {n: torch.empty(shapes[n.replace("v", "k")], device=dev, dtype=torch.uint8) for n in ("k", "v", "ks", "vs")}
    per = max(1, (1 << 27) // (hkv * B * d))
    for n in "kv":
        for at in range(0, n_pages, per):
            m = min(per, n_pages - at)
            x = torch.randn((m, hkv, B, d), generator=gen, device=dev)
            code, nibbles = _quantise(x * gain if n == "k" else x)
            cache[n][at:at + m] = _packed(nibbles)
            cache[n + "s"][at:at + m] = code.transpose(2, 3)
    return cache


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(dev).manual_seed(seed)
    s = {"c": c}
    b, hq, hkv, d, rows, t = c["batch"], c["hq"], c["hkv"], c["d"], c["rows"], TYPES[c["dtype"]]
    if c["kind"] in ("tables", "store", "step"):
        start, n = _lengths(c, gen, dev)
        table, free, n_pages = _pages(c, gen, dev, start, rows)
        s.update(q_start=start, q_len=n, table=table, free=free, n_pages=n_pages,
                 slots=torch.empty((b, rows), device=dev, dtype=torch.int32), kv_len=torch.empty((b,), device=dev, dtype=torch.int32),
                 n_taken=torch.empty((1,), device=dev, dtype=torch.int32))
    if c["kind"] in ("rope", "rope_grad"):
        start, n = _lengths(c, gen, dev)
        s.update(_rope_inputs(c, gen, dev), q_start=start, q_len=n if c["ragged"] else None)
        s["q"], s["k"], _ = _fused(c, gen, dev, (hq, hkv, hkv), t)
        if c["kind"] == "rope":
            s["q_out"] = torch.zeros((b, hq, rows, d), device=dev, dtype=t)
            s["k_out"] = torch.zeros((b, hkv, rows, d), device=dev, dtype=t)
        else:
            s["dq_out"] = torch.randn((b, hq, rows, d), generator=gen, device=dev).to(t)
            s["dk_out"] = torch.randn((b, hkv, rows, d), generator=gen, device=dev).to(t)
            # the gradients go where the projection's own gradient is formed
            whole = torch.zeros((b, rows, (hq + 2 * hkv) * d), device=dev, dtype=t)
            s["dq"], s["dk"], _ = [x.unflatten(2, (-1, d)).transpose(1, 2) for x in whole.split([hq * d, hkv * d, hkv * d], dim=2)]
    elif c["kind"] == "store":
        s["k"], s["v"] = _fused(c, gen, dev, (hkv, hkv), t)
        s["k"] = s["k"].contiguous()                       # (keys come out of the rotation, values out of the projection)
        full = torch.zeros((s["n_pages"], hkv, c["block"], d // 2), device=dev, dtype=torch.uint8)
        scale = torch.zeros((s["n_pages"], hkv, d // 32, c["block"]), device=dev, dtype=torch.uint8)
        s["cache"] = (full, full.clone(), scale, scale.clone())
        s["table"], s["slots"] = _plain_tables(s)[:2]
        s["k_rows"] = torch.zeros((b, hkv, rows, d), device=dev, dtype=t)
        s["v_rows"] = torch.zeros((b, hkv, rows, d), device=dev, dtype=t)
    elif c["kind"] == "decode":
        lens = torch.randint(c["len_lo"], c["len_hi"] + 1, (b,), generator=gen, device=dev, dtype=torch.int32)
        lens[: c["idle"]] = 0
        table, _, n_pages = _pages(c, gen, dev, lens, 0)
        s.update(kv_len=lens, table=table, q=torch.randn((b, hq, d), generator=gen, device=dev).to(t))
        f = _filled_cache(c, gen, dev, n_pages)
        s["cache"] = (f["k"], f["v"], f["ks"], f["vs"])
    elif c["kind"] == "step":
        s.update(_rope_inputs(c, gen, dev))
        s["q"], s["k"], s["v"] = _fused(c, gen, dev, (hq, hkv, hkv), t)
        s["q_out"] = torch.zeros((b, hq, rows, d), device=dev, dtype=t)
        s["k_out"] = torch.zeros((b, hkv, rows, d), device=dev, dtype=t)
        f = _filled_cache(c, gen, dev, s["n_pages"])
        s["cache"] = (f["k"], f["v"], f["ks"], f["vs"])
    if c["kind"] in ("decode", "step"):
        s["o"] = torch.empty((b, hq, d), device=dev, dtype=t)
        s["lse"] = torch.empty((b, hq), device=dev, dtype=torch.float32)
    if c["kind"] in ("rope_grad", "decode", "step"):
        s["workspace"] = {}                                # (made by the first pass, kept as a program keeps it)
    return s


# ---- the library's calls ----------------------------------------------------------------------------------------------
def _own(s):
    from paper_2503_03588_amd import binding as pa
    c = s["c"]
    pat = pa.Pattern(c["block"], c["window"], c["sink"])
    if c["kind"] in ("tables", "step"):
        pa.page_tables(pat, s["q_start"], s["q_len"], s["free"], s["table"], s["n_pages"], c["rows"], slots=s["slots"],
                       kv_len=s["kv_len"], n_taken=s["n_taken"])
        if c["kind"] == "tables":
            return s["table"], s["slots"], s["kv_len"], s["n_taken"]
    if c["kind"] in ("rope", "step"):
        pa.qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], q_start=s["q_start"], q_len=s["q_len"],
                        eps=EPS, interleaved=c["interleaved"], q_out=s["q_out"], k_out=s["k_out"])
        if c["kind"] == "rope":
            return s["q_out"], s["k_out"]
    if c["kind"] == "rope_grad":
        ws = s["workspace"]
        if "it" not in ws:
            ws["it"] = pa.qk_norm_rope_backward_workspace(c["batch"], c["hq"], c["hkv"], c["rows"], c["d"])
        return pa.qk_norm_rope_backward(s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], s["dq_out"], s["dk_out"],
                                        q_start=s["q_start"], q_len=s["q_len"], eps=EPS, interleaved=c["interleaved"], dq=s["dq"],
                                        dk=s["dk"], workspace=ws["it"])
    if c["kind"] == "store":
        pa.cache_store_q4(pat, s["k"], s["v"], s["cache"], s["slots"])
        return pa.cache_load_q4(pat, s["cache"], s["table"], c["rows"], start=s["q_start"], length=s["q_len"], k=s["k_rows"],
                                v=s["v_rows"])
    ws, stride = s["workspace"], s["table"].shape[1]
    if "it" not in ws:
        ws["it"] = pa.decode_paged_q4_workspace(pat, c["batch"], c["hq"], c["hkv"], c["d"], stride * c["block"])
    if c["kind"] == "step":
        pa.cache_store_q4(pat, s["k_out"], s["v"], s["cache"], s["slots"])
        q = s["q_out"].view(c["batch"], c["hq"], c["d"])
    else:
        q = s["q"]
    o, lse = pa.decode_paged_q4(pat, q, s["cache"], s["table"], s["kv_len"], o=s["o"], lse=s["lse"], workspace=ws["it"])
    return (o, lse, s["table"], s["slots"], s["kv_len"]) if c["kind"] == "step" else (o, lse)


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _plain_tables(s):
    """(table, slots, kv_len, number of pages taken)"""
    c = s["c"]
    B, rows, table, free = c["block"], c["rows"], s["table"], s["free"]
    stride, cap, dev = table.shape[1], table.shape[1] * c["block"], table.device
    start = s["q_start"].long().clamp(0, cap)
    n = torch.minimum(s["q_len"].long().clamp(0, rows), cap - start)
    held, need = (start + B - 1) // B, (start + n + B - 1) // B
    base = torch.cumsum(need - held, 0) - (need - held)
    padded = torch.cat([free.long(), torch.full((1,), -1, device=dev)])
    j = torch.arange(stride, device=dev)[None]
    which = (base[:, None] + j - held[:, None]).clamp(0, free.numel())
    table = torch.where((j >= held[:, None]) & (j < need[:, None]), padded[which], table.long())
    r = torch.arange(rows, device=dev)[None]
    pos = start[:, None] + r
    page = table.gather(1, (pos // B).clamp(max=stride - 1))
    good = (r < n[:, None]) & (page >= 0) & (page < s["n_pages"])
    slots = torch.where(good, page * B + pos % B, -1)
    return table.int(), slots.int(), (start + n).int(), (need - held).sum().int().view(1)


def _cos_sin(s):
    """cos and sin of every row's angles [b, 1, rows, rot/2]; the angles in 64 bits, far positions having many turns."""
    r = torch.arange(s["c"]["rows"], device=s["inv_freq"].device)
    pos = s["q_start"].double()[:, None] + r
    angle = pos[:, None, :, None] * s["inv_freq"].double()
    return angle.cos().float(), angle.sin().float()


def _turned(x, cos, sin, c):
    """The rotation of the first `rot` components."""
    rot = c["rot"]
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(s, x, w, like):
    c = s["c"]
    cos, sin = _cos_sin(s)
    x = x.float()
    y = _turned(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float(), cos, sin, c).to(like.dtype)
    return torch.where(_row_is_there(s), y, like)


def _row_is_there(s):
    """[b, 1, rows, 1]: the rows behind a sequence's last one stay as they were"""
    r = torch.arange(s["c"]["rows"], device=s["q_start"].device)
    n = s["q_len"] if s["q_len"] is not None else torch.full_like(s["q_start"], s["c"]["rows"])
    return (r < n[:, None])[:, None, :, None]


def _plain_rope_grad(s, x, w, dy, like):
    c = s["c"]
    cos, sin = _cos_sin(s)
    there = _row_is_there(s)
    x, w = x.float(), w.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    normed = x * r
    du = _turned(dy.float(), cos, -sin, c)
    dw = torch.where(there, du * normed, 0.0).sum((0, 1, 2))
    dn = du * w
    dx = r * (dn - normed * (dn * normed).mean(-1, keepdim=True))
    return torch.where(there, dx.to(like.dtype), like), dw


def _quantise(x):
    """Scale codes [..., d/32] and 4-bit codes [..., d] of fp32 values."""
    g = x.unflatten(-1, (-1, 32))
    amax = g.abs().amax(-1)
    bits = amax.view(torch.int32) & 0x7FFFFFFF
    code = (((bits + 0x200000) >> 23) - 2).clamp(0, 252)            # amax's exponent, one more from 1.75 on: 7 is not 6
    bad = bits >= 0x7F800000
    y = torch.where(bad[..., None], 0.0, g * ((254 - code) << 23).view(torch.float32)[..., None])
    a = y.abs()
    n = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    n = n + 8 * torch.signbit(y)
    return torch.where(bad, 255, code).to(torch.uint8), n.to(torch.uint8).flatten(-2)


def _packed(nibbles):
    return nibbles[..., 0::2] | (nibbles[..., 1::2] << 4)


def _values(pages, codes):
    """fp32 values [..., d] of packed rows [..., d/2] with the scale codes [..., d/32]."""
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=pages.device)
    x = torch.stack([grid[(pages & 15).int()], grid[(pages >> 4).int()]], -1).flatten(-2)
    bits = torch.where(codes == 0, 0x400000, codes.int() << 23)                    # 2^(code - 127)
    scale = torch.where(codes == 255, math.nan, bits.view(torch.float32))
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _plain_store(s, k, v):
    """Rows into the pages, as the slots say."""
    c, slots = s["c"], s["slots"].long()
    here = torch.nonzero(slots.flatten() >= 0)[:, 0]
    at = slots.flatten()[here]
    page, off = at // c["block"], at % c["block"]
    data, scales = s["cache"][:2], s["cache"][2:]
    _put(k, here, page, off, data[0], scales[0])
    _put(v, here, page, off, data[1], scales[1])


def _put(x, here, page, off, data, scales):
    code, nibbles = _quantise(x.transpose(1, 2).flatten(0, 1)[here].float())       # [tokens, hkv, d]
    data[page, :, off] = _packed(nibbles)
    scales[page, :, :, off] = code


def _plain_load(s, data, scales, like):
    c = s["c"]
    r = torch.arange(c["rows"], device=data.device)
    pos = s["q_start"].long()[:, None] + r
    page = s["table"].long().gather(1, (pos // c["block"]).clamp(max=s["table"].shape[1] - 1)).clamp(0, data.shape[0] - 1)
    x = _values(data[page, :, pos % c["block"]], scales[page, :, :, pos % c["block"]])      # [b, rows, hkv, d]
    return torch.where(_row_is_there(s), x.transpose(1, 2).to(like.dtype), like)


def _attended(c, kv_len, stride):
    """The attended blocks of every sequence's query, ascending [b, n]; -1 behind the last one."""
    j = torch.arange(stride, device=kv_len.device)[None]
    i = ((kv_len.long() - 1) // c["block"])[:, None]
    dist = i - j
    on = (dist >= 0) & ((dist < c["window"]) | ((dist & (dist - 1)) == 0) | (j < c["sink"]))
    most = min(stride, c["window"] + c["sink"] + stride.bit_length() + 1)
    at = torch.where(on, j, stride).sort(1).values[:, :most]
    return torch.where(at < stride, at, -1)


def _plain_decode(s, q, kv_len):
    c, B, d = s["c"], s["c"]["block"], s["c"]["d"]
    b, hq, hkv = c["batch"], c["hq"], c["hkv"]
    kd, vd, ks, vs = s["cache"]
    blocks = _attended(c, kv_len, s["table"].shape[1])
    page = s["table"].long().gather(1, blocks.clamp(min=0)).clamp(0, kd.shape[0] - 1)
    k = _values(kd[page], ks[page].transpose(3, 4)).permute(0, 2, 1, 3, 4).flatten(2, 3)     # [b, hkv, tokens, d]
    v = _values(vd[page], vs[page].transpose(3, 4)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    pos = (blocks[:, :, None] * B + torch.arange(B, device=q.device)).flatten(1)
    on = ((blocks >= 0).repeat_interleave(B, 1) & (pos < kv_len[:, None]))[:, None, None]
    x = torch.matmul(q.float().view(b, hkv, hq // hkv, d), k.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = torch.where(on, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, torch.where(on[:, :, 0, :, None], v, 0.0)) / torch.where(total == 0, 1.0, total)
    return o.view(b, hq, d).to(q.dtype), (top + torch.log(total)).view(b, hq)


def _plain(s):
    c = s["c"]
    if c["kind"] == "tables":
        return _plain_tables(s)
    if c["kind"] == "rope":
        return _plain_rope(s, s["q"], s["q_weight"], s["q_out"]), _plain_rope(s, s["k"], s["k_weight"], s["k_out"])
    if c["kind"] == "rope_grad":
        dq, dqw = _plain_rope_grad(s, s["q"], s["q_weight"], s["dq_out"], s["dq"])
        dk, dkw = _plain_rope_grad(s, s["k"], s["k_weight"], s["dk_out"], s["dk"])
        return dq, dk, dqw, dkw
    if c["kind"] == "store":
        _plain_store(s, s["k"], s["v"])
        return _plain_load(s, s["cache"][0], s["cache"][2], s["k_rows"]), _plain_load(s, s["cache"][1], s["cache"][3], s["v_rows"])
    if c["kind"] == "decode":
        return _plain_decode(s, s["q"], s["kv_len"])
    table, slots, kv_len, _ = _plain_tables(s)
    s = {**s, "table": table, "slots": slots}
    q = _plain_rope(s, s["q"], s["q_weight"], s["q_out"])
    k = _plain_rope(s, s["k"], s["k_weight"], s["k_out"])
    _plain_store(s, k, s["v"])
    o, lse = _plain_decode(s, q[:, :, 0], kv_len)
    return o, lse, table, slots, kv_len


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def _mean_attended(c):
    """Attended tokens of a row of mean length (every block whole)."""
    n = max(1, (c["len_lo"] + c["len_hi"]) // 2)
    i = (n - 1) // c["block"]
    far = sum(1 for j in range(i + 1) if i - j < c["window"] or (i - j) & (i - j - 1) == 0 or j < c["sink"])
    return min(n, far * c["block"])


def work(case):
    c = case
    b, hq, hkv, d, rows = c["batch"], c["hq"], c["hkv"], c["d"], c["rows"]
    size = 4 if c["dtype"] == "f32" else 2
    tokens = b * rows // (2 if c["ragged"] else 1)
    packed = d // 2 + d // 32
    w = {"bytes": 0, "flops": 0}
    if c["kind"] in ("tables", "step"):
        w["bytes"] += 12 * b + 4 * b * rows + 12 * (tokens // c["block"] + 1)
    if c["kind"] in ("rope", "rope_grad", "step"):
        passes = 3 if c["kind"] == "rope_grad" else 2
        w["bytes"] += passes * tokens * (hq + hkv) * d * size
        w["flops"] += (30 if passes == 3 else 10) * tokens * (hq + hkv) * d
    if c["kind"] == "store":
        w["bytes"] += 2 * 2 * tokens * hkv * (2 * d + packed)
        w["flops"] += 8 * tokens * hkv * d
    if c["kind"] == "step":
        w["bytes"] += 2 * tokens * hkv * (2 * d + packed)
    if c["kind"] in ("decode", "step"):
        att = b * _mean_attended(c)
        w["bytes"] += 2 * att * hkv * packed + 4 * b * hq * d
        w["flops"] += 4 * att * hq * d
    return w


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def _exact_rope(s, x, w):
    """The rotation as a product of complex numbers."""
    c, d, rot = s["c"], s["c"]["d"], s["c"]["rot"]
    u = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + EPS) * w
    turns = s["q_start"].double().view(-1, 1, 1, 1) + torch.arange(c["rows"], device=x.device, dtype=torch.float64).view(1, 1, -1, 1)
    turn = torch.polar(torch.ones((), device=x.device, dtype=torch.float64), turns * s["inv_freq"].double())
    if c["interleaved"]:
        z = torch.view_as_real(torch.view_as_complex(u[..., :rot].unflatten(-1, (rot // 2, 2)).contiguous()) * turn).flatten(-2)
    else:
        z = torch.complex(u[..., : rot // 2].contiguous(), u[..., rot // 2: rot].contiguous()) * turn
        z = torch.cat((z.real, z.imag), -1)
    return torch.cat((z, u[..., rot:]), -1)


def _exact_rows(s, y):
    if s["q_len"] is None:
        return y
    behind = torch.arange(s["c"]["rows"], device=y.device) >= s["q_len"][:, None]
    return y.masked_fill(behind[:, None, :, None], 0.0)


def _power_of_two(e):
    return ((e + 1023) << 52).view(torch.float64)


def _exact_4bit(x):
    """The nearest of the sixteen values, in units of the group's power of two; the even code where two are equally near."""
    grid = torch.tensor(E2M1, device=x.device, dtype=torch.float64)
    out = torch.empty_like(x)
    step = max(1, (1 << 24) // x[0].numel())
    for at in range(0, x.shape[0], step):
        g = x[at:at + step].unflatten(-1, (-1, 32))
        amax = g.abs().amax(-1, keepdim=True)
        m, e = torch.frexp(amax)                                   # amax = m 2^e, m in [1/2, 1)
        e = torch.where(m >= 0.875, e + 1, e) - 3
        e = torch.where(amax == 0, -127, e).clamp(-127, 125)
        unit = _power_of_two(e.long())
        far = ((g.abs() / unit)[..., None] - grid).abs()
        far[..., 1::2] = far[..., 1::2] * (1 + 1e-12) + 1e-300     # odd codes lose ties
        y = grid[far.argmin(-1)] * torch.sign(g) * unit
        out[at:at + step] = torch.where(torch.isfinite(amax), y, math.nan).flatten(-2)
    return out


def _exact_decode(c, q, k, v, n):
    """One sequence: q [hq, d], and all its keys and values [hkv, n, d]."""
    B, i = c["block"], (n - 1) // c["block"]
    blocks = [j for j in range(i + 1) if i - j < c["window"] or bin(i - j).count("1") == 1 or j < c["sink"]]
    at = torch.cat([torch.arange(j * B, min((j + 1) * B, n), device=q.device) for j in blocks])
    x = torch.bmm(q.view(c["hkv"], -1, c["d"]), k[:, at].transpose(1, 2).contiguous()) * c["d"] ** -0.5
    return torch.bmm(torch.softmax(x, -1), v[:, at]).view(c["hq"], c["d"]), torch.logsumexp(x, -1).view(c["hq"])


def _exact_pages(s, which, blocks_of_table):
    """Values [hkv, blocks * B, d] of the pages of one sequence."""
    data, codes = s["cache"][which], s["cache"][2 + which]
    pages = blocks_of_table.long()
    lo_hi = torch.stack((data[pages] % 16, data[pages] // 16), -1).flatten(-2).long()
    signs = 1.0 - 2.0 * (lo_hi // 8).double()
    x = signs * torch.tensor(E2M1, device=data.device, dtype=torch.float64)[lo_hi % 8]
    unit = _power_of_two(codes[pages].long() - 127)
    return (x * unit.transpose(2, 3).repeat_interleave(32, -1)).transpose(0, 1).flatten(1, 2)


def exact(case, seed):
    c = case
    if c["kind"] == "tables":
        return None                                                # whole numbers
    s = prepare(case, seed)
    if c["kind"] == "rope":
        return tuple(_exact_rows(s, _exact_rope(s, s[n].double(), s[n + "_weight"].double())) for n in "qk")
    if c["kind"] == "rope_grad":
        dx, dw = [], []
        for n in "qk":
            x, w = s[n].double().requires_grad_(), s[n + "_weight"].double().requires_grad_()
            dy = _exact_rows(s, s["d" + n + "_out"].double())
            gx, gw = torch.autograd.grad(_exact_rope(s, x, w), (x, w), dy)
            dx.append(gx)
            dw.append(gw)
        return (*dx, *dw)
    if c["kind"] == "store":
        return tuple(_exact_rows(s, _exact_4bit(s[n].double())) for n in "kv")
    b, hq, d, B = c["batch"], c["hq"], c["d"], c["block"]
    o = torch.zeros((b, hq, d), device="cuda", dtype=torch.float64)
    lse = torch.full((b, hq), -math.inf, device="cuda", dtype=torch.float64)
    if c["kind"] == "decode":
        for i, n in enumerate(s["kv_len"].tolist()):
            if n:
                pages = s["table"][i, : -(-n // B)]
                o[i], lse[i] = _exact_decode(c, s["q"][i].double(), _exact_pages(s, 0, pages), _exact_pages(s, 1, pages), n)
        return o, lse
    # The step: every call's outputs in the type that the next call takes.  (No value for the log-sum-exp: a key that lies
    # between two of the 4-bit values within the error of 32 bits may be held as either.)
    q = _exact_rope(s, s["q"].double(), s["q_weight"].double()).to(torch.bfloat16).double()
    k = _exact_4bit(_exact_rope(s, s["k"].double(), s["k_weight"].double()).to(torch.bfloat16).double())
    v = _exact_4bit(s["v"].double())
    for i, (start, n) in enumerate(zip(s["q_start"].tolist(), s["q_len"].tolist())):
        if start + n:
            pages = s["table"][i, : -(-start // B)]
            keys = torch.cat((_exact_pages(s, 0, pages)[:, :start], k[i, :, :n]), 1)
            values = torch.cat((_exact_pages(s, 1, pages)[:, :start], v[i, :, :n]), 1)
            o[i], lse[i] = _exact_decode(c, q[i, :, 0], keys, values, start + n)
    return o, None, None, None, None
