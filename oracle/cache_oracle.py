"""fp64 CPU oracle of the rotation, of the cache's 8-bit rows and of the attention over cached rows, from their formulas (numpy only).

    rotation   z = w n, n = r x, r = (mean x^2 + eps)^-1/2;  (y_a, y_b) = (z_a cos t - z_b sin t, z_b cos t + z_a sin t)
               dz = R^T dy;  dw = sum dz n;  dx = r (w dz - n mean(w dz n))
    rows       blocks of 32: the smallest 2^e, e >= -117, with top / 2^e <= 448; e4m3(x / 2^e), to nearest even
    attention  s_ij = scale q_i.k_j or cap tanh(scale q_i.k_j / cap) over the keys that row i takes; o_i = sum softmax(s_i)_j v_j

Beside every value stands an elementwise bound on what rounding may do to it when norms, functions, scores and sums are fp32 (unit u32 = 2^-24;
sums of n terms n u32) and outputs are rounded to the type once (unit u), weights as operands twice or more (what a rounding leaves is a further operand):
    r          er = (d / 2 + 8) u32 of itself: d squares, the root;   cos, sin   ec = 6 u32 + 2^-51 |angle|, absolutely
    y          (|z_a| + |z_b|) (ec + er + 5 u32) + u |y|
    dz         e_dz = (|dy_a| + |dy_b|) (ec + 3 u32)
    dw         sum |n| (e_dz + |dz| (er + (min(terms, 64) + 10) u32)) + u |dw| + terms 2^-150 (sums of tiny terms): a lane adds up some of its workgroup's
               rows, 64 of them at most wherever this is compared, eight steps add the lanes of a workgroup, and workgroups are joined in 64 bits
    dx         r (|w| e_dz + |n| e_m + (2 er + 8 u32) (|w dz| + |n m|)) + u |dx|,   m the mean, e_m = mean |n| (|w| e_dz + |w dz| (er + (d + 4) u32))
    scores     ds = 2 (d + 8) u32 max_j (scale sum |q||k| + |lse|) + 20 u32 max_j |s|   (of a weight; the last with a cap, whose tanh is off by less than 10 u32 of itself)
    o          (u^2 + ds + (n + 1) u32) sum p|v| + u |o|   (bf16: weights are three operands, u^2 stands for less than u32)
fp16 adds half a step of its subnormal numbers (weights are lifted by 2^6 before they meet them).
"""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}      # half a step of the subnormal numbers (fp32: one)


# ---- rotation ---------------------------------------------------------------------------------------
def pairs(rot, neighbours):
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if neighbours else (p, p + rot // 2)


def angles(pos, freq, axis):
    """(batch, row, pair), pos (axes, batch, row) whole numbers."""
    lead = np.zeros(len(freq), int) if axis is None else np.asarray(axis, int)
    return np.moveaxis(np.asarray(pos, np.float64)[lead], 0, -1) * np.asarray(freq, np.float64) if len(freq) else np.zeros(pos.shape[1:] + (0,))


def _turn(x, a, b, cos, sin):
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def rotate(kind, x, angle, neighbours=False, eps=None, weight=None, dy=None, row_len=None):
    """x (batch, row, head, feature).  Returns (values, bounds): dicts with y and, with dy, dx and (with a weight) dw."""
    u, tiny = UNIT[kind], TINY[kind]
    x = np.asarray(x, np.float64).copy()
    d = x.shape[-1]
    live = np.ones(x.shape[:2], bool)
    if row_len is not None:
        live = np.arange(x.shape[1])[None, :] < np.clip(np.asarray(row_len), 0, x.shape[1])[:, None]
    dead = ~live[:, :, None, None]
    x = np.where(dead, 0.0, x)
    a, b = pairs(2 * angle.shape[-1], neighbours)
    cos, sin = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
    ec = 6 * U32 + 2.0 ** -51 * np.abs(angle)[:, :, None]
    w = np.ones(d) if weight is None else np.asarray(weight, np.float64)
    n, r, er = x, np.ones(x.shape[:3] + (1,)), 0.0
    if eps is not None:
        er = (d / 2 + 8) * U32
        with np.errstate(divide="ignore", invalid="ignore"):
            r = ((x * x).mean(-1, keepdims=True) + eps) ** -0.5
            n = x * r
    n = np.where(dead, 0.0, n)

    def spread(m, e):                                        # |a| + |b| of a pair, times what its functions add
        out = np.zeros_like(m)
        out[..., a] = out[..., b] = (m[..., a] + m[..., b]) * e
        return out

    z = n * w
    y = _turn(z, a, b, cos, sin)
    both = spread(np.abs(z), 1.0)
    plain = np.ones(d, bool)
    plain[a] = plain[b] = False
    err = spread(np.abs(z), ec) + np.where(plain, np.abs(z), both) * (er + 5 * U32) + u * np.abs(y) + tiny
    val, lim = {"y": y}, {"y": np.where(dead, 0.0, err)}
    if dy is None:
        return val, lim
    dy = np.where(dead, 0.0, np.asarray(dy, np.float64))
    dz = _turn(dy, a, b, cos, -sin)
    e_dz = spread(np.abs(dy), ec + 3 * U32)
    if weight is not None:
        terms = x.shape[0] * x.shape[1] * x.shape[2]
        val["dw"] = (dz * n).sum((0, 1, 2))
        lim["dw"] = (np.abs(n) * (e_dz + np.abs(dz) * (er + (min(terms, 64) + 10) * U32))).sum((0, 1, 2)) + u * np.abs(val["dw"]) + tiny
        lim["dw"] += terms * 2.0 ** -150                     # an addition of fp32 numbers is off by half a step of their subnormal ones
    dx, e = dz, e_dz + 3 * U32 * np.abs(dz)
    if eps is not None:
        wz = w * dz
        m = (wz * n).mean(-1, keepdims=True)
        e_m = (np.abs(n) * (np.abs(w) * e_dz + np.abs(wz) * (er + (d + 4) * U32))).mean(-1, keepdims=True)
        dx = r * (wz - n * m)
        e = r * (np.abs(w) * e_dz + np.abs(n) * e_m + (2 * er + 8 * U32) * (np.abs(wz) + np.abs(n * m)))
    val["dx"] = np.where(dead, 0.0, dx)
    lim["dx"] = np.where(dead, 0.0, e + u * np.abs(dx) + tiny)
    return val, lim


# ---- 8-bit rows -------------------------------------------------------------------------------------
def e4m3(x):
    """Nearest 8-bit float (even of two), |x| <= 448; NaN stays."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.where(x == 0, 1.0, x))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.round(x / step) * step


def quantise(x, kind="bf16"):
    """(values, exponents) of rows: what the cache holds of x (..., width) of a type, and e of its blocks (..., blocks).  What would round beyond
    the type's largest value (256 2^e, e = 120 or, in fp16, 8) is the largest below."""
    x = np.asarray(x, np.float64)
    held, exps = np.empty_like(x), []
    for c in range(0, x.shape[-1], 32):
        block = x[..., c:c + 32]
        fine = np.isfinite(block)
        top = np.where(fine, np.abs(block), 0.0).max(-1, keepdims=True)
        m, e = np.frexp(top)                                 # top = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
        e = np.where(top == 0, 0, np.maximum(e - 9 + (m > 0.875), -117))
        q = e4m3(np.where(fine, block, 0.0) * np.exp2(-e.astype(float)))
        q = np.where(e == (8 if kind == "f16" else 120), np.clip(q, -240, 240), q)
        held[..., c:c + 32] = np.where(fine, q * np.exp2(e.astype(float)), np.nan)
        exps.append(e[..., 0])
    return held, np.stack(exps, -1)


# ---- attention --------------------------------------------------------------------------------------
def taken(n, nq, total, causal=True, window=0):
    """(nq, n) keys that the rows of a sequence of n keys take; row i stands at n - nq + i."""
    p = n - nq + np.arange(nq)[:, None]
    j = np.arange(total)[None, :]
    keep = np.broadcast_to(j < n, (nq, total)).copy()
    if causal:
        keep &= j <= p
    if window:
        keep &= j > p - window
    return keep


def attend(kind, Q, K, V, scale, k_len, q_len=None, causal=True, window=0, cap=0.0, there=None, once=False):
    """Q (batch, nq, heads, d); K, V (batch, rows, kv_heads, .) of every sequence; there (batch, rows): rows whose page is there;
    once: weights are rounded once only, as bbmm_attend does.  Returns (values, bounds): dicts with o and lse."""
    u, tiny = UNIT[kind], TINY[kind]
    B, nq, H, d = Q.shape
    total, HK, dv = K.shape[1], K.shape[2], V.shape[3]
    G = H // HK
    val = {"o": np.zeros((B, nq, H, dv)), "lse": np.full((B, H, nq), -np.inf)}
    err = {"o": np.zeros((B, nq, H, dv)), "lse": np.zeros((B, H, nq))}
    for b in range(B):
        n = min(max(int(k_len[b]), 0), total)
        ni = nq if q_len is None else min(max(int(q_len[b]), 0), nq)
        keep = taken(n, ni, total, causal, window)
        if there is not None:
            keep &= there[b][None, :]
        for i in range(ni):
            at = np.nonzero(keep[i])[0]
            if not len(at):
                continue
            for h in range(H):
                q, k, v = Q[b, i, h], K[b, at, h // G], V[b, at, h // G]
                s = scale * (k @ q)
                big = scale * (np.abs(k) @ np.abs(q)).max()
                if cap:
                    s = cap * np.tanh(s / cap)
                top = s.max()
                lse = top + np.log(np.exp(s - top).sum())
                p = np.exp(s - lse)
                ds = 2 * (d + 8) * U32 * (big + abs(lse)) + (20 * U32 * np.abs(s).max() if cap else 0.0)
                o = p @ v
                val["o"][b, i, h], val["lse"][b, h, i] = o, lse
                err["o"][b, i, h] = ((u if once else u * u) + ds + (len(at) + 1) * U32) * (p @ np.abs(v)) + u * np.abs(o) + tiny * (1 + 2.0 ** -4 * np.abs(v).sum(0))
                err["lse"][b, h, i] = ds + (len(at) + 4) * U32 + 4 * U32 * abs(lse)
    return val, err
