"""Norm and rotation of queries and keys, the paged cache that keys and values live in, and the attention of new tokens that
reads it: measured cases, their inputs, the plain forms and the definitions in 64 bits.

    rotation    z = x w (mean x^2 + eps)^-1/2;  (y_a, y_b) = (z_a cos t - z_b sin t, z_b cos t + z_a sin t) for every pair
                (a, b) of the first `rot` features, t = pos[axis of the pair] freq[pair]
    cache       rows of pages, in their own type or in e4m3 with a power of two for every 32 features: the smallest 2^e,
                e >= -117, by which the block's largest value becomes at most 448; e + 127 is held in a byte
    attention   s_ij = cap tanh(scale q_i.k_j / cap) over the keys p_i - window < j <= p_i, p_i = k_len - nq + i;
                o_i = sum_j exp(s_ij - lse_i) v_j, lse_i = log sum_j exp(s_ij)

Kinds of cases: "rotate" (forward), "train" (rotation and all gradients), "write" (new rows into the pages), "cache" (new rows
written, the whole of every sequence read back) and "attend".  Rows of Q, K, V, O: (batch, row, head, feature).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
DEVICE = "cuda:0"
EPS = 1e-6


# ---- cases ------------------------------------------------------------------------------------------
def _rot(name, kind, dtype, batch, rows, heads, kv_heads, d, rot=None, norm=True, axes=1, neighbours=False, start=0):
    return {"name": name, "kind": kind, "dtype": dtype, "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads, "d": d,
            "rot": d if rot is None else rot, "norm": norm, "axes": axes, "neighbours": neighbours, "start": start}


def _cache(name, kind, dtype, held, batch, new, total, kv_heads, d, dv=None, page=64, ragged=False):
    return {"name": name, "kind": kind, "dtype": dtype, "held": held, "batch": batch, "new": new, "total": total,
            "kv_heads": kv_heads, "d": d, "dv": dv or d, "page": page, "ragged": ragged}


def _att(name, dtype, held, batch, heads, kv_heads, nq, nk, d, dv=None, page=64, ragged=False, window=0, cap=0.0):
    return {"name": name, "kind": "attend", "dtype": dtype, "held": held, "batch": batch, "heads": heads, "kv_heads": kv_heads,
            "nq": nq, "total": nk, "d": d, "dv": dv or d, "page": page, "ragged": ragged, "window": window, "cap": cap}


def listed():
    return [
        # the next token of one request, far into its text: the call's own latency
        _rot("rotate_one_bf16", "rotate", "bf16", 1, 1, 32, 8, 128, start=100000),
        # a prompt on its way into the cache
        _rot("rotate_prompt_bf16", "rotate", "bf16", 1, 8192, 32, 8, 128),
        # patches of two videos: time, height and width, neighbouring pairs, no norm
        _rot("rotate_axes_f16", "rotate", "f16", 2, 2309, 16, 16, 80, norm=False, axes=3, neighbours=True),
        # a training step of a layer with shared heads
        _rot("train_bf16", "train", "bf16", 4, 2048, 16, 4, 128),
        # a training step at full precision, half of the features rotated
        _rot("train_f32", "train", "f32", 2, 500, 8, 8, 64, rot=32),
        # the newest row of eight requests into their pages
        _cache("write_one_bf16", "write", "bf16", "same", 8, 1, 1000, 8, 128, page=16, ragged=True),
        # a chunk of a prompt into 8-bit pages, and everything back for the chunk's own attention
        _cache("cache_chunk_e4m3", "cache", "bf16", "e4m3", 4, 2048, 8192, 8, 128),
        # one request of a few keys: the call's own latency
        _att("attend_one_short_bf16", "bf16", "same", 1, 4, 4, 1, 77, 64, page=16),
        # single tokens of eight requests of unequal length over a long memory with shared heads
        _att("attend_one_long_bf16", "bf16", "same", 8, 32, 8, 1, 32773, 128, ragged=True),
        # many requests over 8-bit pages
        _att("attend_one_long_e4m3", "bf16", "e4m3", 16, 32, 8, 1, 65536, 128, ragged=True),
        # many short requests, every head its own keys, a window over the latest ones and small pages
        _att("attend_window_f16", "f16", "same", 64, 16, 16, 1, 3001, 64, page=16, ragged=True, window=1024),
        # three proposed tokens of two requests at full precision, capped scores, pages that no tile fits
        _att("attend_few_f32", "f32", "same", 2, 8, 8, 3, 10000, 64, page=20, cap=30.0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "rotate", "train", "train", "write", "cache", "attend", "attend", "attend"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    size = SIZE[dtype]
    kv = rng.choice([1, 2, 4, 8, 12])
    batch = rng.randint(1, 16)
    d = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128])
    if kind in ("rotate", "train"):
        heads = kv * rng.choice([1, 1, 2, 4])
        rows = rng.choice([1, 1, spread(2, 8000), spread(2, 8000)])
        while size * batch * rows * (heads + kv) * d > 1.0e8:
            batch, rows = max(1, batch // 2), max(1, rows * 3 // 4)
        axes = rng.choice([1, 1, 2, 3])
        rot = d if rng.random() < 0.7 else 2 * rng.randint(1, d // 2)
        return _rot(None, kind, dtype, batch, rows, heads, kv, d, rot, rng.random() < 0.7, axes, rng.random() < 0.4,
                    rng.choice([0, spread(1, 1000000)]))
    held = rng.choice(["same", "e4m3"]) if kind != "write" else "same"
    dv = d if rng.random() < 0.8 else rng.choice([16, 32, 64, 128])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256, 1, 20])
    ragged = rng.random() < 0.6
    if kind in ("write", "cache"):
        total = spread(1, 10000)
        new = min(total, rng.choice([1, spread(1, 4000)]))
        while size * batch * total * kv * (d + dv) > 1.5e8:
            batch, total = max(1, batch // 2), max(1, total * 3 // 4)
            new = min(new, total)
        return _cache(None, kind, dtype, held, batch, new, total, kv, d, dv, page, ragged)
    heads = kv * rng.choice([1, 1, 2, 4, 8])
    nq = rng.choice([1, 1, 1, 1, 2, 3, 5, 8])
    total = max(nq, spread(1, 100000))
    batch = spread(1, 64)
    while size * batch * total * kv * (d + dv) > (3e8 if dtype == "f32" else 1e9):
        if batch > 1:
            batch = batch * 3 // 4
        else:
            total = max(nq, total * 3 // 4)
    return _att(None, dtype, held, batch, heads, kv, nq, total, d, dv, page, ragged, rng.choice([0, 0, 0, spread(16, 8000)]),
                rng.choice([0.0, 0.0, 50.0]))


def _lengths(case):
    """Rows of every sequence: all of them, or spread evenly below the longest, in no order of size."""
    b, n = case["batch"], case["total"]
    least = case["nq"] if case["kind"] == "attend" else case["new"]
    return [max(least, n - (i * 7919 % b) * n // (b + 1)) if case["ragged"] else n for i in range(b)]


# ---- inputs -----------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, spread=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32) * spread).to(t)

    st = {"case": case}
    b, d, kv = case["batch"], case["d"], case["kv_heads"]
    if case["kind"] in ("rotate", "train"):
        rows, heads, half = case["rows"], case["heads"], case["rot"] // 2
        # queries, keys and values come out of one product, side by side
        qkv = normal(b, rows, heads + 2 * kv, d)
        st["q"], st["k"] = qkv[:, :, :heads], qkv[:, :, heads:heads + kv]
        st["q_weight"] = st["k_weight"] = None
        if case["norm"]:
            st["q_weight"], st["k_weight"] = (1 + normal(d, spread=0.3).float()).to(t), (1 + normal(d, spread=0.3).float()).to(t)
        st["freq"] = 10000.0 ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / max(half, 1))
        at = torch.arange(rows, device=DEVICE) + case["start"]
        if case["axes"] == 1:
            pos = at[None, None].expand(1, b, rows)
        else:                                   # frames of 24 x 24 patches
            pos = torch.stack([at // 576, at // 24 % 24, at % 24][-case["axes"]:])[:, None].expand(case["axes"], b, rows)
        st["pos"] = pos.contiguous()
        st["axis"] = [p * case["axes"] // max(half, 1) for p in range(half)]
        if case["kind"] == "train":
            st["dq"], st["dk"] = normal(b, rows, heads, d), normal(b, rows, kv, d)
        return st
    lens = _lengths(case)
    page, dv, e4m3 = case["page"], case["dv"], case["held"] == "e4m3"
    per = [(n + page - 1) // page for n in lens]
    pages = sum(per) + 3
    places = torch.randperm(pages, generator=g, device=DEVICE).tolist()
    table, at = [], 0
    for n in per:
        table.append(places[at:at + n] + [-1] * (max(per) - n))
        at += n
    st["table"] = torch.tensor(table, device=DEVICE, dtype=torch.int32)
    # pages of (head, row, feature), rows from 16 bytes to 16 bytes; seen as (page, row, head, feature)
    step = 16 if e4m3 else 16 // SIZE[case["dtype"]]
    for name, width in (("k", d), ("v", dv)):
        values = normal(pages, kv, page, width)
        if e4m3:
            values, st[name + "_exp"] = _to_e4m3(values)
        held = torch.zeros(pages, kv, page, (width + step - 1) // step * 16, device=DEVICE, dtype=torch.uint8)
        held[..., :width * values.element_size()] = values.view(torch.uint8)
        held = held.view(values.dtype)
        st[name + "_pages"] = held[..., :width].transpose(1, 2)
    if case["kind"] == "attend":
        st["q"] = normal(b, case["nq"], case["heads"], d)
        st["scale"] = d ** -0.5
        st["k_len"] = torch.tensor(lens, device=DEVICE, dtype=torch.int32)
    else:
        kv_new = normal(b, case["new"], kv, d + dv)
        st["k"], st["v"] = kv_new[..., :d], kv_new[..., d:]
        st["start"] = torch.tensor([n - case["new"] for n in lens], device=DEVICE, dtype=torch.int32)
        st["length"] = torch.tensor(lens, device=DEVICE, dtype=torch.int32)
    return st


# ---- the plain forms --------------------------------------------------------------------------------
def _power(e):
    """2^e in 32 bits, from its bits: -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _to_e4m3(x):
    """Values in e4m3 and their blocks' exponent bytes, four a row."""
    width = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -width % 32)).unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))         # m in [1/2, 1): the largest value is 2 m 2^(e - 1)
    e = e - 9 + (m > 0.875).int()
    e = torch.where(m == 0, 0, e.clamp(min=-117))
    q = (x * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    q = q.flatten(-2).view(torch.uint8)[..., :width].contiguous().view(torch.float8_e4m3fn)
    return q, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, 4 - e.shape[-1]), value=127)


def _from_e4m3(q, exps):
    """The values in 32 bits: q (..., width) and the exponent bytes (..., 4) of its rows."""
    scale = _power(exps.int() - 127).repeat_interleave(32, -1)[..., :q.shape[-1]]
    return q.float() * scale


def _sequences(st, name):
    """Rows of all sequences in 32 bits, (batch, rows of the longest's pages, head, feature); missing pages read page 0."""
    at = st["table"].long().clamp(min=0)
    values = st[name + "_pages"][at] if st["case"]["held"] == "same" else st[name + "_pages"].view(torch.uint8)[at]
    if st["case"]["held"] == "e4m3":
        values = _from_e4m3(values.view(torch.float8_e4m3fn), st[name + "_exp"].transpose(1, 2)[at])
    return values.flatten(1, 2).float()


def _turn(case, x, cos, sin):
    """Pairs of the first `rot` features turned by their angles: cos and sin (batch, row, 1, pair)."""
    rot = case["rot"]
    if case["neighbours"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _rotate_plain(st):
    case, t = st["case"], st["q"].dtype
    axis = torch.tensor(st["axis"], device=DEVICE, dtype=torch.int64)
    angle = (st["pos"][axis].double() * st["freq"][:, None, None]).permute(1, 2, 0)[:, :, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {}
    for name in ("q", "k"):
        x, w = st[name].float(), 1.0
        r = 1.0
        if case["norm"]:
            w = st[name + "_weight"].float()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        out[name] = _turn(case, n * w, cos, sin).to(t)
        if case["kind"] == "train":
            dz = _turn(case, st["d" + name].float(), cos, -sin)
            dn = dz * w
            if case["norm"]:
                out["d" + name + "_weight"] = (dz * n).sum((0, 1, 2)).to(t)
                dn = r * (dn - n * (dn * n).mean(-1, keepdim=True))
            out["d" + name] = dn.to(t)
    return out


def _write_plain(st):
    case = st["case"]
    at = st["start"].long()[:, None] + torch.arange(case["new"], device=DEVICE)
    page = torch.gather(st["table"].long(), 1, at // case["page"])
    row = at % case["page"]
    for name in ("k", "v"):
        if case["held"] == "same":
            st[name + "_pages"][page, row] = st[name]
        else:
            q, exps = _to_e4m3(st[name])
            st[name + "_pages"].view(torch.uint8)[page, row] = q.view(torch.uint8)
            st[name + "_exp"].transpose(1, 2)[page, row] = exps


def _read_plain(st):
    case, t = st["case"], st["k"].dtype
    there = torch.arange(case["total"], device=DEVICE)[None, :] < st["length"][:, None]
    return {name: torch.where(there[:, :, None, None], _sequences(st, name)[:, :case["total"]], 0.0).to(t) for name in ("k", "v")}


def _attend_plain(st):
    case, t = st["case"], st["q"].dtype
    b, nq, kv = case["batch"], case["nq"], case["kv_heads"]
    group = case["heads"] // kv
    k, v = (_sequences(st, name).transpose(1, 2).contiguous() for name in ("k", "v"))
    q = st["q"].float().view(b, nq, kv, group, case["d"]).permute(0, 2, 4, 3, 1).reshape(b, kv, case["d"], group * nq)
    s = torch.matmul(k, q.contiguous()) * st["scale"]
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    at = st["k_len"][:, None].long() - nq + torch.arange(nq, device=DEVICE)
    j = torch.arange(k.shape[2], device=DEVICE)[None, :, None]
    keep = j <= at[:, None]
    if case["window"]:
        keep &= j > at[:, None] - case["window"]
    s = torch.where(keep[:, None, :, None], s.unflatten(3, (group, nq)), -math.inf)
    m = s.amax(2, keepdim=True)
    e = torch.exp(s - m)
    total = e.sum(2, keepdim=True)
    p = (e / total).flatten(3).transpose(2, 3).contiguous()
    o = torch.matmul(p, v).view(b, kv, group, nq, case["dv"])
    lse = (m + torch.log(total))[:, :, 0].reshape(b, case["heads"], nq)
    return {"o": o.permute(0, 3, 1, 2, 4).reshape(b, nq, case["heads"], case["dv"]).to(t), "lse": lse}


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind in ("rotate", "train"):
        return _rotate_plain(st)
    if kind == "attend":
        return _attend_plain(st)
    _write_plain(st)
    return {"k": st["k_pages"], "v": st["v_pages"]} if kind == "write" else _read_plain(st)


# ---- the framework's calls --------------------------------------------------------------------------
_context = None


def _run_own(st):
    global _context
    from paper_1809_11165_amd import binding
    if _context is None:
        _context = binding.Context(0)
    case, ctx = st["case"], _context
    if case["kind"] in ("rotate", "train"):
        rot = binding.Rotation(st["q"], st["k"], st["pos"], st["freq"], axis=st["axis"], neighbours=case["neighbours"],
                               eps=EPS if case["norm"] else None, q_weight=st["q_weight"], k_weight=st["k_weight"])
        q, k = ctx.bbmm_rotate(rot)
        out = {"q": q, "k": k}
        if case["kind"] == "train":
            dq, dk, dq_weight, dk_weight = ctx.bbmm_rotate_grad(rot, st["dq"], st["dk"])
            out |= {"dq": dq, "dk": dk}
            if case["norm"]:
                out |= {"dq_weight": dq_weight, "dk_weight": dk_weight}
        return out
    cache = binding.Cache(st["k_pages"], st["v_pages"], st["table"], k_exp=st.get("k_exp"), v_exp=st.get("v_exp"))
    if case["kind"] == "attend":
        o, lse = ctx.bbmm_attend_cache(binding.CachedAttention(cache, st["q"], st["k_len"], scale=st["scale"], causal=True,
                                                               window=case["window"], cap=case["cap"]))
        return {"o": o, "lse": lse}
    ctx.bbmm_cache_write(cache, st["k"], st["v"], start=st["start"])
    if case["kind"] == "write":
        return {"k": st["k_pages"], "v": st["v_pages"]}
    k, v = ctx.bbmm_cache_read(cache, case["total"], length=st["length"], dtype=st["k"].dtype)
    return {"k": k, "v": v}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    size, b, d, kv = SIZE[case["dtype"]], case["batch"], case["d"], case["kv_heads"]
    if case["kind"] in ("rotate", "train"):
        values = b * case["rows"] * (case["heads"] + kv) * d
        few = 8 * case["axes"] * b * case["rows"] + 4 * case["rot"] + (2 * size * d if case["norm"] else 0)
        if case["kind"] == "rotate":
            return {"bytes": 2 * size * values + few, "flops": 7 * values}
        return {"bytes": 4 * size * values + few + (2 * size * d if case["norm"] else 0), "flops": 20 * values}
    lens, dv = _lengths(case), case["dv"]

    def row(width):
        return size * width if case["held"] == "same" else width + (width + 31) // 32

    held = kv * (row(d) + row(dv))
    if case["kind"] == "attend":
        reach = case["window"] + case["nq"] - 1 if case["window"] else case["total"]
        keys = sum(min(n, reach) for n in lens)
        rows = b * case["nq"] * case["heads"]
        return {"bytes": keys * held + rows * (size * (d + dv) + 4), "flops": 2 * case["nq"] * case["heads"] * keys * (d + dv)}
    moved = b * case["new"] * (size * kv * (d + dv) + held)
    if case["kind"] == "cache":
        moved += (sum(lens) - b * case["new"]) * held + b * case["total"] * size * kv * (d + dv)
    return {"bytes": moved, "flops": 0}


# ---- the definition in 64 bits ----------------------------------------------------------------------
def _rotate_exact(st, out):
    case = st["case"]
    rot, half = case["rot"], case["rot"] // 2
    first = [2 * p if case["neighbours"] else p for p in range(half)]
    second = [2 * p + 1 if case["neighbours"] else p + half for p in range(half)]
    lead = torch.tensor(st["axis"], device=DEVICE, dtype=torch.int64)
    angle = torch.stack([st["pos"][int(a)].double() * f for a, f in zip(lead, st["freq"])], -1)      # (batch, row, pair)
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    for name in ("q", "k"):
        x = st[name].double()
        n, r, w = x, None, torch.ones(case["d"], device=DEVICE, dtype=torch.float64)
        if case["norm"]:
            w = st[name + "_weight"].double()
            r = (x.square().sum(-1, keepdim=True) / case["d"] + EPS) ** -0.5
            n = x * r

        def turned(z, by):
            y = z.clone()
            c = torch.complex(z[..., first], z[..., second]) * by
            y[..., first], y[..., second] = c.real, c.imag
            return y

        out[name] = turned(n * w, turn)
        if case["kind"] == "train":
            dz = turned(st["d" + name].double(), turn.conj())
            if case["norm"]:
                out["d" + name + "_weight"] = (dz * n).flatten(0, 2).sum(0)
                dz = dz * w
                dz = r * dz - x * r ** 3 * (dz * x).sum(-1, keepdim=True) / case["d"]
            out["d" + name] = dz
    return out


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held_exact(x):
    """What e4m3 pages keep of 64-bit values: steps of 2^-3 of a value's power of two, of 2^-9 units below 2^-6 units."""
    y = torch.zeros_like(x)
    for c in range(0, x.shape[-1], 32):
        block = x[..., c:c + 32]
        top = block.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448))
        e = torch.where(top > _exact_power(e) * 448, e + 1, e)
        e = torch.where(top <= _exact_power(e - 1) * 448, e - 1, e).clamp(min=-117)
        unit = _exact_power(e)
        power = torch.floor(torch.log2(torch.clamp(block.abs() / unit, min=2.0 ** -6)))
        step = _exact_power(power - 3) * unit
        y[..., c:c + 32] = torch.round(block / step) * step
    return y


def _row_exact(st, name, i, n):
    """Rows 0 .. n of sequence i from its pages in 64 bits (row, head, feature)."""
    case = st["case"]
    at = torch.arange(n, device=DEVICE)
    page, row = st["table"][i].long()[at // case["page"]], at % case["page"]
    if case["held"] == "same":
        return st[name + "_pages"][page, row].double()
    q = st[name + "_pages"].view(torch.uint8)[page, row].view(torch.float8_e4m3fn).double()
    for c in range(0, q.shape[-1], 32):
        q[..., c:c + 32] *= _exact_power(st[name + "_exp"][page, :, row][..., c // 32].long() - 127)[..., None]
    return q


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("rotate", "train"):
        return _rotate_exact(st, {})
    lens, out = _lengths(case), {}
    if case["kind"] == "attend":
        b, h, nq, group = case["batch"], case["heads"], case["nq"], case["heads"] // case["kv_heads"]
        o = torch.zeros(b, nq, h, case["dv"], device=DEVICE, dtype=torch.float64)
        lse = torch.full((b, h, nq), -math.inf, device=DEVICE, dtype=torch.float64)
        for i, n in enumerate(lens):
            low = max(0, n - nq - case["window"] + 1) if case["window"] else 0
            k, v = (_row_exact(st, name, i, n)[low:] for name in ("k", "v"))
            for r in range(nq):
                p = n - nq + r
                lo = max(low, p - case["window"] + 1) if case["window"] else low
                s = torch.einsum("jhd,hgd->hgj", k[lo - low:p + 1 - low], st["q"][i, r].double().view(-1, group, case["d"])) * st["scale"]
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                lse[i, :, r] = torch.logsumexp(s, 2).flatten()
                o[i, r] = torch.einsum("hgj,jhd->hgd", torch.softmax(s, 2), v[lo - low:p + 1 - low]).flatten(0, 1)
        return {"o": o, "lse": lse}
    for name in ("k", "v"):
        if case["kind"] == "write":
            pages = st[name + "_pages"].double()
            for i, n in enumerate(lens):
                at = torch.arange(n - case["new"], n, device=DEVICE)
                pages[st["table"][i].long()[at // case["page"]], at % case["page"]] = st[name][i].double()
            out[name] = pages
            continue
        rows = torch.zeros(case["batch"], case["total"], case["kv_heads"], st[name].shape[3], device=DEVICE, dtype=torch.float64)
        for i, n in enumerate(lens):
            rows[i, :n] = _row_exact(st, name, i, n)
            new = st[name][i].double()
            rows[i, n - case["new"]:n] = _held_exact(new) if case["held"] == "e4m3" else new
        out[name] = rows
    return out
