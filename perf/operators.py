"""Attention of queries to inputs of another length, and the learned bias by buckets of the position difference:
measured cases, their inputs, the plain forms and the definitions in 64 bits.

    s_ij = scale q_i.k_j + T[h, bucket(j - i - start_b)]   over the keys j < k_len_b that the mask keeps
    o_i  = sum_j exp(s_ij - lse_i) v_j,   lse_i = log sum_j exp(s_ij)   (nothing left: o_i = 0, lse_i = -inf)

Kinds of cases: "attend" (forward only), "train" (forward and all gradients), "bias" (the bias as a matrix) and
"bias_grad" (the table's gradient from the matrix's).  Rows of Q, O: (batch, query, head, feature).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEVICE = "cuda:0"


# ---- cases ------------------------------------------------------------------------------------------
def _att(name, kind, dtype, batch, heads, kv_heads, nq, nk, d, dv=None, buckets=0, far=0, two_sided=True, start=0,
         ragged=False, mask=False):
    return {"name": name, "kind": kind, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "nq": nq,
            "nk": nk, "d": d, "dv": dv or d, "buckets": buckets, "far": far, "two_sided": two_sided, "start": start,
            "ragged": ragged, "mask": mask}


def _bias(name, kind, dtype, batch, heads, nq, nk, buckets, far, two_sided=True, start=0):
    return {"name": name, "kind": kind, "dtype": dtype, "batch": batch, "heads": heads, "nq": nq, "nk": nk,
            "buckets": buckets, "far": far, "two_sided": two_sided, "start": start}


def listed():
    return [
        # one query over a short memory: the call's own latency
        _att("attend_one_short_bf16", "attend", "bf16", 1, 4, 4, 1, 77, 64, buckets=32, far=128),
        # single tokens of eight requests of unequal length over a long memory with shared heads
        _att("attend_one_long_bf16", "attend", "bf16", 8, 32, 8, 1, 32773, 128, ragged=True),
        # a few test inputs against 10 000 training inputs in fp32, one request, learned bias at the end of the memory
        _att("attend_few_long_f32", "attend", "f32", 1, 8, 8, 3, 10000, 64, buckets=32, far=128, start=9997),
        # a padded batch of ordinary length, key mask and bias
        _att("attend_batch_f16", "attend", "f16", 4, 16, 16, 1000, 1537, 64, buckets=32, far=128, ragged=True, mask=True),
        # the largest: long queries over a longer memory
        _att("attend_large_bf16", "attend", "bf16", 2, 16, 16, 4096, 10000, 128, buckets=32, far=128),
        # a training step of an ordinary encoder-decoder layer
        _att("train_batch_bf16", "train", "bf16", 8, 12, 12, 512, 640, 64, buckets=32, far=128, ragged=True),
        # a training step at full precision on regression-sized inputs
        _att("train_f32", "train", "f32", 2, 8, 8, 500, 1000, 64, buckets=32, far=128),
        # a training step over a long memory with shared heads
        _att("train_long_bf16", "train", "bf16", 2, 16, 4, 2048, 8192, 128),
        # the bias alone, as a small matrix and as one that fills the memory bus
        _bias("bias_small_f32", "bias", "f32", 1, 8, 128, 200, 32, 128),
        _bias("bias_large_bf16", "bias", "bf16", 1, 16, 4096, 8192, 32, 128),
        # its gradient, summed over the batch that the bias was broadcast to
        _bias("bias_grad_small_f32", "bias_grad", "f32", 2, 8, 128, 200, 32, 128),
        _bias("bias_grad_large_bf16", "bias_grad", "bf16", 4, 16, 1024, 2048, 32, 128),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most_flops, most_bytes = 600e9, 0.9e9
    kind = rng.choice(["attend_few", "attend_few", "attend", "attend", "train", "train", "bias", "bias_grad"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    size = 4 if dtype == "f32" else 2
    buckets = rng.choice([8, 16, 32, 64])
    two = rng.random() < 0.7
    far = spread(buckets, 512)
    if kind in ("bias", "bias_grad"):
        heads, batch = rng.randint(1, 20), 1 if kind == "bias" else rng.randint(1, 4)
        nq, nk = spread(1, 4000), spread(1, 8000)
        while size * batch * heads * nq * nk > most_bytes:
            nq = max(1, nq // 2)
        return _bias(None, kind, dtype, batch, heads, nq, nk, buckets, far, two, rng.choice([0, 0, rng.randint(-500, 5000)]))
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 1, 1, 2, 4])
    d = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128])
    dv = d if rng.random() < 0.8 else rng.choice([16, 32, 64, 128])
    batch = rng.randint(1, 8)
    if kind == "attend_few":
        nq, nk = rng.choice([1, 1, 1, 2, 3, 7, 16, 31]), spread(1, 50000)
    else:
        nq, nk = spread(33, 4000), spread(20, 10000)
    cost = (1 if kind != "train" else 3.5) * (8 if dtype == "f32" else 1)
    while 2 * batch * heads * nq * nk * (d + dv) * cost > most_flops or size * batch * kv * nk * (d + dv) > most_bytes:
        if batch > 1:
            batch -= 1
        elif nk > 2 * nq:
            nk = nk * 3 // 4
        else:
            nq = max(1, nq * 3 // 4)
    bias = rng.random() < 0.6
    return _att(None, "train" if kind == "train" else "attend", dtype, batch, heads, kv, nq, nk, d, dv, buckets if bias else 0,
                far if bias else 0, two, rng.choice([0, max(0, nk - nq)]) if bias else 0, rng.random() < 0.5, rng.random() < 0.25)


def _edges(buckets, far, two_sided):
    """Ascending distances at which the bucket changes: unit steps up to half of a side's buckets, then equal steps of
    the logarithm up to `far`, from whole numbers (x^n against powers: no rounding at a border)."""
    side = buckets // 2 if two_sided else buckets
    near = max(1, side // 2)
    edges = list(range(1, near + 1))
    n = side - near
    for k in range(1, n):
        x = edges[-1] + 1
        while x ** n < near ** (n - k) * max(far, near + 1) ** k:
            x += 1
        edges.append(x)
    return edges[:side - 1]


def _k_len(case):
    """Lengths of the batch's keys: a padded batch loses up to half of them."""
    b, nk = case["batch"], case["nk"]
    return [nk - (i * nk) // (2 * b) for i in range(b)]


# ---- inputs -----------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, spread=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32) * spread).to(t)

    st = {"case": case}
    if case["buckets"]:
        st["edges"] = _edges(case["buckets"], case["far"], case["two_sided"])
        n = len(st["edges"]) + 1
        st["table"] = normal(case["heads"], 2 * n if case["two_sided"] else n)
    if case["kind"] in ("bias", "bias_grad"):
        if case["kind"] == "bias_grad":
            st["dB"] = normal(case["batch"], case["heads"], case["nq"], case["nk"])
        return st
    b, nq, nk = case["batch"], case["nq"], case["nk"]
    st["q"] = normal(b, nq, case["heads"], case["d"])
    st["k"] = normal(b, nk, case["kv_heads"], case["d"])
    st["v"] = normal(b, nk, case["kv_heads"], case["dv"])
    st["scale"] = case["d"] ** -0.5
    st["k_len"] = torch.tensor(_k_len(case), device=DEVICE, dtype=torch.int32) if case["ragged"] else None
    st["mask"] = None
    if case["mask"]:
        st["mask"] = torch.rand(b, nk, generator=g, device=DEVICE) < 0.9
    st["start"] = None
    if case["buckets"]:
        st["start"] = torch.full((b,), case["start"], device=DEVICE, dtype=torch.int64)
    if case["kind"] == "train":
        st["do"] = normal(b, nq, case["heads"], case["dv"])
    return st


# ---- the plain forms --------------------------------------------------------------------------------
def _bucket_line(edges, two_sided):
    """Bucket of every difference from -e to e, e the last edge (further ones share its bucket)."""
    e = edges[-1] if edges else 1
    r = torch.arange(-e, e + 1, device=DEVICE)
    dist = r.abs() if two_sided else (-r).clamp(min=0)
    at = torch.tensor(edges, device=DEVICE, dtype=torch.int64)
    n = (dist[:, None] >= at[None, :]).sum(1)
    return (n + (r > 0) * (len(edges) + 1) if two_sided else n), e


def _bias_of(table, edges, two_sided, start, nq, nk):
    """(batch or 1, head, nq, nk) in 32 bits."""
    line, e = _bucket_line(edges, two_sided)
    i = torch.arange(nq, device=DEVICE)[None, :, None]
    j = torch.arange(nk, device=DEVICE)[None, None, :]
    n = line[(j - i - start[:, None, None]).clamp(-e, e) + e]
    return table.float()[:, n].transpose(0, 1)


def _keep(st, nk):
    keep = None
    if st["k_len"] is not None:
        keep = torch.arange(nk, device=DEVICE)[None, :] < st["k_len"][:, None]
    if st["mask"] is not None:
        keep = st["mask"] if keep is None else keep & st["mask"]
    return keep


def _scores(st):
    case = st["case"]
    group = case["heads"] // case["kv_heads"]
    keep = _keep(st, case["nk"])
    k, v = st["k"].float(), st["v"].float()
    if keep is not None:
        k = torch.where(keep[:, :, None, None], k, 0.0)
        v = torch.where(keep[:, :, None, None], v, 0.0)
    q = st["q"].float().transpose(1, 2).contiguous()
    k = k.transpose(1, 2).repeat_interleave(group, 1).contiguous()
    v = v.transpose(1, 2).repeat_interleave(group, 1).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    if case["buckets"]:
        s = s + _bias_of(st["table"], st["edges"], case["two_sided"], st["start"], case["nq"], case["nk"])
    if keep is not None:
        s = torch.where(keep[:, None, None, :], s, -math.inf)
    return q, k, v, s


def _attend_plain(st):
    q, k, v, s = _scores(st)
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(s - m)
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    return q, k, v, p, torch.matmul(p, v), (m + torch.log(total)).squeeze(3)


def _train_plain(st):
    case, t = st["case"], st["q"].dtype
    group = case["heads"] // case["kv_heads"]
    q, k, v, p, o, lse = _attend_plain(st)
    do = st["do"].float().transpose(1, 2).contiguous()
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(3, keepdim=True))
    dq = torch.matmul(ds, k) * st["scale"]
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * st["scale"]
    shape = (case["batch"], case["kv_heads"], group, case["nk"], -1)
    out = {"o": o.transpose(1, 2).contiguous().to(t), "lse": lse, "dq": dq.transpose(1, 2).contiguous().to(t),
           "dk": dk.view(shape).sum(2).transpose(1, 2).contiguous().to(t),
           "dv": dv.view(shape).sum(2).transpose(1, 2).contiguous().to(t)}
    if case["buckets"]:
        out["dtable"] = _table_sums(ds, st["edges"], case["two_sided"], st["start"], st["table"].shape[1]).to(t)
    return out


def _table_sums(ds, edges, two_sided, start, buckets):
    """Sums of (batch, head, nq, nk) by bucket: along the diagonals first (rows turned over and padded to a width of
    nq + nk, read again one column narrower: diagonals become columns), then the diagonals of each bucket."""
    b, h, nq, nk = ds.shape
    wide = torch.nn.functional.pad(ds.flip(2), (0, nq)).reshape(b, h, -1)[:, :, :nq * (nq + nk - 1)]
    by_difference = wide.view(b, h, nq, nq + nk - 1).sum(2, dtype=torch.float64)
    line, e = _bucket_line(edges, two_sided)
    r = torch.arange(nq + nk - 1, device=DEVICE)[None, :] - (nq - 1) - start[:, None]
    of = line[r.clamp(-e, e) + e][:, :, None] == torch.arange(buckets, device=DEVICE)
    return torch.matmul(by_difference, of.double()).sum(0)


def _run_plain(st):
    case = st["case"]
    if case["kind"] == "attend":
        o, lse = _attend_plain(st)[-2:]
        return {"o": o.transpose(1, 2).contiguous().to(st["q"].dtype), "lse": lse}
    if case["kind"] == "train":
        return _train_plain(st)
    start = torch.tensor([case["start"]], device=DEVICE)
    if case["kind"] == "bias":
        return _bias_of(st["table"], st["edges"], case["two_sided"], start, case["nq"], case["nk"])[0].to(st["table"].dtype)
    return _table_sums(st["dB"].float(), st["edges"], case["two_sided"], start, st["table"].shape[1]).to(st["dB"].dtype)


# ---- the framework's calls --------------------------------------------------------------------------
_context = None


def _run_own(st):
    global _context
    from paper_1809_11165_amd import binding
    if _context is None:
        _context = binding.Context(0)
    case, ctx = st["case"], _context
    if case["kind"] == "bias":
        return ctx.bbmm_bucket_bias(st["table"], st["edges"], case["nq"], case["nk"], two_sided=case["two_sided"],
                                    start=case["start"])
    if case["kind"] == "bias_grad":
        return ctx.bbmm_bucket_bias_grad(st["dB"], st["edges"], two_sided=case["two_sided"], start=case["start"])
    att = binding.Attention(st["q"], st["k"], st["v"], scale=st["scale"], k_len=st["k_len"], key_mask=st["mask"],
                            table=st.get("table"), edges=st.get("edges"), two_sided=case["two_sided"], q_start=st["start"])
    o, lse = ctx.bbmm_attend(att)
    if case["kind"] == "attend":
        return {"o": o, "lse": lse}
    dq, dk, dv, dtable = ctx.bbmm_attend_grad(att, o, lse, st["do"])
    out = {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if dtable is not None:
        out["dtable"] = dtable
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    h, nq, nk = case["heads"], case["nq"], case["nk"]
    table = size * h * case["buckets"]
    if case["kind"] == "bias":
        return {"bytes": size * h * nq * nk + table, "flops": 0}
    if case["kind"] == "bias_grad":
        return {"bytes": size * case["batch"] * h * nq * nk + table, "flops": case["batch"] * h * nq * nk}
    b, kv, d, dv = case["batch"], case["kv_heads"], case["d"], case["dv"]
    keys = sum(_k_len(case)) if case["ragged"] else b * nk
    q, o, k, v, lse = size * b * h * nq * d, size * b * h * nq * dv, size * keys * kv * d, size * keys * kv * dv, 4 * b * h * nq
    moved = q + k + v + o + lse + table + (b * nk if case["mask"] else 0)
    flops = 2 * h * nq * keys * (d + dv)
    if case["kind"] == "train":
        moved += q + o + size * b * nk * kv * (d + dv) + table      # dO in; dQ, dK, dV and the table's gradient out
        flops += 2 * h * nq * keys * (3 * d + 2 * dv)
    return {"bytes": moved, "flops": flops}


# ---- the definition in 64 bits ----------------------------------------------------------------------
def _bucket_exact(case, edges, start):
    """Bucket of every pair, counted edge by edge."""
    r = (torch.arange(case["nk"], device=DEVICE).view(1, -1) - torch.arange(case["nq"], device=DEVICE).view(-1, 1)) - start
    dist = torch.maximum(r, -r) if case["two_sided"] else torch.maximum(-r, torch.zeros_like(r))
    n = torch.zeros_like(r)
    for e in edges:
        n += dist >= e
    if case["two_sided"]:
        n += torch.where(r >= 1, len(edges) + 1, 0)
    return n


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "bias":
        n = _bucket_exact(case, st["edges"], case["start"])
        return torch.stack([row[n] for row in st["table"].double()])
    if case["kind"] == "bias_grad":
        n = _bucket_exact(case, st["edges"], case["start"]).reshape(-1)
        rows = []
        for h in range(case["heads"]):
            out = torch.zeros(st["table"].shape[1], device=DEVICE, dtype=torch.float64)
            rows.append(out.index_add_(0, n, st["dB"][:, h].double().sum(0).reshape(-1)))
        return torch.stack(rows)
    train, group = case["kind"] == "train", case["heads"] // case["kv_heads"]
    b, h, nq = case["batch"], case["heads"], case["nq"]

    def zeros(*shape):
        return torch.zeros(*shape, device=DEVICE, dtype=torch.float64)

    out = {"o": zeros(b, nq, h, case["dv"]), "lse": zeros(b, h, nq)}
    if train:
        out |= {"dq": zeros(*st["q"].shape), "dk": zeros(*st["k"].shape), "dv": zeros(*st["v"].shape)}
        if case["buckets"]:
            out["dtable"] = zeros(*st["table"].shape)
    for i in range(b):
        some = torch.ones(case["nk"], device=DEVICE, dtype=torch.bool)
        if st["k_len"] is not None:
            some[int(st["k_len"][i]):] = False
        if st["mask"] is not None:
            some &= st["mask"][i]
        at = some.nonzero()[:, 0]
        if not len(at):
            out["lse"][i] = -math.inf
            continue
        n = _bucket_exact(case, st["edges"], int(st["start"][i]))[:, at] if case["buckets"] else None
        for j in range(h):
            q, k, v = st["q"][i, :, j].double(), st["k"][i, at, j // group].double(), st["v"][i, at, j // group].double()
            s = (q @ k.T.contiguous()) * st["scale"]
            if n is not None:
                s += st["table"][j].double()[n]
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            o = p @ v
            out["o"][i, :, j], out["lse"][i, j] = o, lse
            if train:
                do = st["do"][i, :, j].double()
                ds = do @ v.T.contiguous()
                ds = p * (ds - (p * ds).sum(1, keepdim=True))
                out["dv"][i, at, j // group] += p.T.contiguous() @ do
                out["dq"][i, :, j] = (ds @ k) * st["scale"]
                out["dk"][i, at, j // group] += (ds.T.contiguous() @ q) * st["scale"]
                if n is not None:
                    out["dtable"][j].index_add_(0, n.reshape(-1), ds.reshape(-1))
    return out
