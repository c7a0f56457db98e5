"""fp64 CPU oracle of the attention and of its bucketed bias, from their formulas (numpy only).

    s_ij = scale q_i.k_j + T[h, bucket(j - i - start_b)]   over j < k_len_b with mask_bj
    o_i  = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij);  nothing left: o_i = 0, lse_i = -inf

`attend` also returns, for every output, an elementwise bound on what rounding may do to it when scores, statistics and sums are
fp32 (unit u32 = 2^-24), weights and dS are rounded to the input type (unit u) as operands, and outputs once:
    scores           ds  = 2 (d + 8) u32 max_j (scale sum |q||k| + |bias| + |lse|)     (relative error of a weight)
    o                (u + ds + n u32) sum p|v| + u |o|
    dP, delta        (d + 8) u32 sum |do||v|,  sum |do| err(o)
    dS               p (ds |dP - delta| + err(dP) + err(delta)),  + u |dS| as an operand
and the last line summed against |k|, |q| or by bucket.  fp16 adds the steps of its subnormal numbers, which operands meet
after their scaling by powers of two.
"""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}          # half a step of the subnormal numbers


def bucket(r, edges, two_sided):
    """Bucket of an integer array of differences."""
    r = np.asarray(r, dtype=np.int64)
    dist = np.abs(r) if two_sided else np.maximum(-r, 0)
    n = np.zeros(r.shape, dtype=np.int64)
    for e in edges:
        n += dist >= e
    return n + ((r > 0) * (len(edges) + 1) if two_sided else 0)


def bias_matrix(table, edges, two_sided, start, nq, nk):
    r = np.arange(nk)[None, :] - np.arange(nq)[:, None] - start
    return np.asarray(table, dtype=np.float64)[:, bucket(r, edges, two_sided)]


def table_grad(dB, edges, two_sided, start):
    """Sums by bucket of dB (batch, head, nq, nk), and the sums of magnitudes."""
    b, h, nq, nk = dB.shape
    n = bucket(np.arange(nk)[None, :] - np.arange(nq)[:, None] - start, edges, two_sided).reshape(-1)
    count = (len(edges) + 1) * (2 if two_sided else 1)
    flat = np.asarray(dB, dtype=np.float64).reshape(b, h, nq * nk)
    out, mag = np.zeros((h, count)), np.zeros((h, count))
    for x in range(h):
        for y in range(b):
            out[x] += np.bincount(n, flat[y, x], count)
            mag[x] += np.bincount(n, np.abs(flat[y, x]), count)
    return out, mag


def attend(kind, Q, K, V, scale, dO=None, q_len=None, k_len=None, mask=None, table=None, edges=(), two_sided=True, start=None):
    """kind: "f32", "f16" or "bf16" (of the rounding bounds).  Arrays as the calls take them, float64.  Returns (values, bounds):
    dicts with o, lse and, with dO, dq, dk, dv and dtable."""
    u, tiny = UNIT[kind], TINY[kind]
    B, nq, H, d = Q.shape
    nk, HK, dv = K.shape[1], K.shape[2], V.shape[3]
    G = H // HK
    val = {"o": np.zeros((B, nq, H, dv)), "lse": np.full((B, H, nq), -np.inf)}
    err = {"o": np.zeros((B, nq, H, dv)), "lse": np.zeros((B, H, nq))}
    if dO is not None:
        for name, x in (("dq", Q), ("dk", K), ("dv", V)):
            val[name], err[name] = np.zeros(x.shape), np.zeros(x.shape)
        if table is not None:
            val["dtable"], err["dtable"] = np.zeros(table.shape), np.zeros(table.shape)
            mag = np.zeros(table.shape)
    big = 0.0
    if dO is not None and kind == "f16":                      # scaling of dS: the largest |do| |v| among what takes part
        def largest(x, n, keep):
            rows = [x[b, :n[b]][keep[b, :n[b]]] for b in range(B)]
            return max([0.0] + [np.sqrt((r ** 2).sum(-1)).max() for r in rows if r.size])
        ql = [nq] * B if q_len is None else [min(max(int(z), 0), nq) for z in q_len]
        kl = [nk] * B if k_len is None else [min(max(int(z), 0), nk) for z in k_len]
        big = largest(dO, ql, np.ones((B, nq), bool)) * largest(V, kl, np.ones((B, nk), bool) if mask is None else mask.astype(bool))
    for b in range(B):
        ni = nq if q_len is None else min(max(int(q_len[b]), 0), nq)
        keep = np.zeros(nk, bool)
        keep[:nk if k_len is None else min(max(int(k_len[b]), 0), nk)] = True
        if mask is not None:
            keep &= mask[b].astype(bool)
        at = np.nonzero(keep)[0]
        if not ni or not len(at):
            continue
        off = 0 if start is None else int(start[b])
        n = bucket(at[None, :] - np.arange(ni)[:, None] - off, edges, two_sided)
        for h in range(H):
            q, k, v = Q[b, :ni, h], K[b, at, h // G], V[b, at, h // G]
            s = scale * (q @ k.T)
            big_s = scale * (np.abs(q) @ np.abs(k).T)
            if table is not None:
                bias = table[h][n]
                s = s + bias
                big_s = big_s + np.where(np.isfinite(bias) & (np.abs(bias) < 1e30), np.abs(bias), 0.0)
            top = s.max(1, keepdims=True)
            some = np.isfinite(top[:, 0])
            p = np.exp(np.where(some[:, None], s - np.where(np.isfinite(top), top, 0.0), -np.inf))
            p = np.where(np.isnan(p), 0.0, p)
            total = p.sum(1, keepdims=True)
            p = p / np.where(total > 0, total, 1.0)
            with np.errstate(divide="ignore"):
                lse = np.where(some, top[:, 0] + np.log(total[:, 0]), -np.inf)
            ds_rel = 2 * (d + 8) * U32 * (big_s.max(1) + np.where(some & (np.abs(lse) < 1e30), np.abs(lse), 0.0))[:, None]
            cnt = len(at)
            o = p @ v
            a = p @ np.abs(v)
            eo = (u + ds_rel + cnt * U32) * a + u * np.abs(o) + tiny * (1 + 2.0 ** -4 * np.abs(v).sum(0)[None, :])
            val["o"][b, :ni, h], err["o"][b, :ni, h] = o, np.where(some[:, None], eo, 0.0)
            val["lse"][b, h, :ni] = lse
            err["lse"][b, h, :ni] = np.where(some, ds_rel[:, 0] + (cnt + 4) * U32 + 4 * U32 * np.abs(lse), 0.0)
            if dO is None:
                continue
            do = np.where(some[:, None], dO[b, :ni, h], 0.0)
            dp = do @ v.T
            delta = (do * o).sum(1, keepdims=True)
            ds = p * (dp - delta)
            p_abs = tiny * 2.0 ** -12
            e_ds = p * (ds_rel * np.abs(dp - delta) + (dv + 8) * U32 * (np.abs(do) @ np.abs(v).T) + (np.abs(do) * eo).sum(1, keepdims=True))
            e_op = e_ds + u * np.abs(ds) + tiny * 2.0 ** -13 * big
            rows = slice(0, ni)
            val["dq"][b, rows, h] = scale * (ds @ k)
            err["dq"][b, rows, h] = scale * ((e_op + cnt * U32 * np.abs(ds)) @ np.abs(k))
            val["dk"][b, at, h // G] += scale * (ds.T @ q)
            err["dk"][b, at, h // G] += scale * ((e_op + G * ni * U32 * np.abs(ds)).T @ np.abs(q))
            val["dv"][b, at, h // G] += p.T @ do
            err["dv"][b, at, h // G] += (p * (u + ds_rel + G * ni * U32) + p_abs).T @ np.abs(do)
            if table is not None:
                m = table.shape[1]
                val["dtable"][h] += np.bincount(n.reshape(-1), ds.reshape(-1), m)
                err["dtable"][h] += np.bincount(n.reshape(-1), e_ds.reshape(-1), m)
                mag[h] += np.bincount(n.reshape(-1), np.abs(ds).reshape(-1), m)
    for name in ("dq", "dk", "dv", "dtable"):
        if name in val:
            err[name] += u * np.abs(val[name]) + tiny
    if "dtable" in val:
        err["dtable"] += (nq + nk) * U32 * mag
    return val, err
