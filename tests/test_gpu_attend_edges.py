"""GPU parity of the attention where rows, scales and biases are out of the ordinary: rows that nothing is left for beside infinities and NaN in
places that count, biases that leave an fp32 lse coarse, gradients of unlike size in fp16, and units of work dealt out over the dies."""
import numpy as np
import pytest

from oracle import attend_oracle as A
from test_gpu_attend import DEV, EDGES, TYPES, _case, _check, _host, _oracle, _rand, _run_and_check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_1809_11165_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("edges", [None, EDGES])
@pytest.mark.parametrize("nq,nk", [(2, 130), (100, 130), (100, 1500)])
def test_queries_of_nan_and_infinities_whose_keys_are_all_masked(ctx, kind, edges, nq, nk):
    """Nothing is left for these rows, whatever the query and the gradient hold: o = 0, lse = -infinity, no part in any gradient."""
    rng = np.random.default_rng(31)
    att, dO = _case(rng, kind, 2, 2, 1, nq, nk, 64, 64, edges=edges, mask=0.7)
    att.key_mask[1] = False
    want = _oracle(kind, att, dO)
    att.Q[1] = float("nan")
    att.Q[1, ::2] = float("inf")
    dO[1] = float("nan")
    O, lse, dQ, dK, dV, dT = _run_and_check(ctx, kind, att, dO, want)
    assert torch.all(O[1] == 0) and torch.all(lse[1] == -float("inf"))
    assert torch.all(dQ[1] == 0) and torch.all(dK[1] == 0) and torch.all(dV[1] == 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("edges", [None, EDGES])
@pytest.mark.parametrize("nq", [3, 100])
def test_queries_whose_scores_are_all_minus_infinity(ctx, kind, edges, nq):
    """An infinite feature of the query makes every kept score -infinity; the masked ones, whatever they are, do not count."""
    rng = np.random.default_rng(32)
    att, dO = _case(rng, kind, 1, 2, 1, nq, 90, 32, 32, edges=edges, mask=0.7)
    att.K[..., 0] = att.K[..., 0].abs() + 0.5
    att.Q[0, 1] = 0
    dO[0, 1] = 0                                           # a row without a part in the gradients, for the oracle
    val, err = _oracle(kind, att, dO)
    for name, x in (("o", 0.0), ("dq", 0.0)):
        val[name][0, 1], err[name][0, 1] = x, 0.0
    val["lse"][0, :, 1], err["lse"][0, :, 1] = -np.inf, 0.0
    att.Q[0, 1, :, 0] = -float("inf")
    _run_and_check(ctx, kind, att, dO, (val, err))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq,nk", [(2, 130), (100, 130), (100, 1500)])
def test_rows_without_keys_are_zero_beside_infinite_values(ctx, kind, nq, nk):
    """Rows behind their length, and rows whose bias excludes every key, where a value that others read is infinite."""
    rng = np.random.default_rng(33)
    att, _ = _case(rng, kind, 1, 2, 2, nq, nk, 64, 64, edges=EDGES, start=[-1], q_len=[nq - 1])
    att.table[:, len(EDGES) + 1:] = -float("inf")          # keys ahead: the first row keeps none
    att.V[0, ::7] = float("inf")
    att.V[0, 3::7] = -float("inf")
    O, lse = ctx.bbmm_attend(att)
    for i in (0, nq - 1):
        assert torch.all(O[0, i] == 0) and torch.all(lse[0, :, i] == -float("inf")), i
    if nq > 2:
        assert torch.isfinite(lse[0, :, 1:nq - 1]).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("nq,nk", [(3, 40), (70, 300), (70, 1500)])
def test_rows_without_keys_have_no_part_in_gradients_beside_infinities(ctx, kind, which, nq, nk):
    """One live row, the rest behind its length: their dQ is zero, and so are the table's buckets that only they could reach."""
    rng = np.random.default_rng(34)
    att, dO = _case(rng, kind, 1, 2, 2, nq, nk, 64, 64, edges=EDGES, q_len=[1])
    getattr(att, which)[0, 2::9] = float("inf")
    O, lse = ctx.bbmm_attend(att)
    dQ, _, _, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    assert torch.all(dQ[0, 1:] == 0)
    assert torch.all(dT[:, 1:len(EDGES) + 1] == 0)         # keys behind the query: none for the row at the first key


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [3, 70, 200])
def test_rows_without_keys_have_no_part_in_gradients_of_infinite_keys(ctx, kind, nq):
    """A key whose infinite feature makes every live row's score -infinity weighs nothing: its dK and dV are zero, whatever rows behind the
    length make of it, and the other keys' are as if it were masked."""
    rng = np.random.default_rng(39)
    att, dO = _case(rng, kind, 1, 2, 2, nq, 90, 64, 64, edges=EDGES, q_len=[nq - 1], mask=1.1)
    att.Q[..., 0] = -att.Q[..., 0].abs() - 0.5
    att.K[0, 5], att.key_mask[0, 5] = 0, False
    val, err = _oracle(kind, att, dO)
    att.K[0, 5, :, 0], att.key_mask = float("inf"), None
    O, lse = ctx.bbmm_attend(att)
    _, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    for name, x in (("o", O), ("lse", lse), ("dk", dK), ("dv", dV), ("dtable", dT)):
        _check(x, val, err, name)
    assert torch.all(dK[0, 5] == 0) and torch.all(dV[0, 5] == 0)


@pytest.mark.parametrize("kind,value", [(k, v) for k in ("f32", "f16", "bf16") for v in (-300.0, -1000.0, -4000.0, -10000.0, -30000.0, -60000.0, -65504.0, 5000.0)])
@pytest.mark.parametrize("nq,nk,dv", [(4, 128, 128), (70, 256, 64), (70, 2048, 128)])
@pytest.mark.parametrize("table", [False, True])
def test_gradients_of_rows_that_a_large_bias_flattens(ctx, kind, value, nq, nk, dv, table):
    """The same bias on every key, from a table beside scores too small to be seen (scale 2^-60) or from a feature that is 1 in Q and the bias in
    K, the others zero: every weight is 1 / nk, a power of two, which all types hold.  Weights recovered from an fp32 lse of that size, rounded on its
    way, are off by a factor common to the row, and so is dV, all of one sign here.  Single elements may be off by a rounding of the result, the
    factor (an eighth of half a step of the type, in fp32 2^-16) and fp32 sums; in their total the roundings, 4 dv different ones of at most u, add up like
    the square root of their number (four deviations)."""
    rng = np.random.default_rng(36)
    att, dO = _case(rng, kind, 4, 2, 1, nq, nk, 32, dv, edges=[1] if table else None)
    dO.abs_()
    if table:
        att.table[:] = value
        att.scale = 2.0 ** -60
        bias = float(att.table[0, 0])
    else:
        att.Q[..., :-1], att.K[..., :-1] = 0, 0
        att.Q[..., -1], att.K[..., -1], att.scale = 1, value, 1.0
        bias = float(att.K[0, 0, 0, -1])
    O, lse = ctx.bbmm_attend(att)
    assert np.allclose(_host(lse), bias + np.log(nk), rtol=6 * A.U32, atol=0)
    got = _host(ctx.bbmm_attend_grad(att, O, lse, dO)[2])
    want = np.repeat(_host(dO).sum((1, 2))[:, None, None], nk, 1) / nk
    u = A.UNIT[kind]
    factor = max(u / 8, 2.0 ** -16) + 2 * nq * A.U32
    assert np.all(np.abs(got - want) <= (u + factor) * want + A.TINY[kind])
    assert abs(got[:, 0].sum() / want[:, 0].sum() - 1) <= factor + 4 * u / np.sqrt(3 * 4 * dv)


@pytest.mark.parametrize("kind,value", [("f32", 3e38), ("f32", 3.4028234663852886e38), ("bf16", 3e38), ("bf16", 3.3895313892515355e38), ("f16", 65504.0)])
@pytest.mark.parametrize("nq", [4, 70])
def test_tables_of_the_highest_value(ctx, kind, value, nq):
    """One bucket at the type's end: its keys share the row, the rest weigh nothing.  What a weight 1 / n and a mean of n values take: a
    rounding of the weight, one of the result, and fp32 sums.  (fp16's largest leaves steps of 2^-7 of a score: scores are kept below.)"""
    rng = np.random.default_rng(35)
    att, dO = _case(rng, kind, 1, 2, 1, nq, 90, 32, 32, edges=EDGES)
    att.scale = 2.0 ** -20
    att.table[:] = 0
    att.table[:, -1] = value                                # keys at least the last edge ahead
    u = A.UNIT[kind]
    O, lse = ctx.bbmm_attend(att)
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    assert torch.isfinite(lse).all() and (lse[:, :, :min(nq, 69)] > min(value, 2.2e38) / 2).all()
    V, D, want_dv, size_dv = _host(att.V)[0, :, 0], _host(dO)[0], np.zeros((90, 32)), np.zeros((90, 32))
    for i in range(nq):
        at = np.arange(90) >= i + EDGES[-1]
        if not at.any():                                    # no key that far ahead
            break
        mean, size = V[at].mean(0), np.abs(V[at]).mean(0)
        assert np.all(np.abs(_host(O)[0, i] - mean) <= (2 * u + 128 * A.U32) * size + A.TINY[kind]), i
        want_dv[at] += D[i].sum(0) / at.sum()
        size_dv[at] += np.abs(D[i]).sum(0) / at.sum()
    if nq == 4:                                             # every row has such keys: dV is theirs alone
        assert np.all(np.abs(_host(dV)[0, :, 0] - want_dv) <= (2 * u + 128 * A.U32) * size_dv + A.TINY[kind])
    for x in (dQ, dK, dT):
        assert torch.isfinite(x).all()


@pytest.mark.parametrize("edges", [None, EDGES])
@pytest.mark.parametrize("nq,nk", [(40, 2000), (300, 2000)])
def test_small_rows_of_dO_beside_large_ones_in_fp16(ctx, edges, nq, nk):
    """Rows of dO at 2^10 and at 2^-10 by turns: the small ones' dS, at weights of 1 / 2000, stay out of fp16's subnormal numbers, so that their dQ is off by
    a rounding of dS, of delta's o and of the result, in the 2-norm of a row one u each."""
    rng = np.random.default_rng(37)
    att, dO = _case(rng, "f16", 1, 2, 1, nq, nk, 64, 64, edges=edges)
    att.scale = 64.0
    att.Q.mul_(2.0 ** -9)
    dO[:, ::2].mul_(2.0 ** 10)
    dO[:, 1::2].mul_(2.0 ** -10)
    val, err = _oracle("f16", att, dO)
    O, lse = ctx.bbmm_attend(att)
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    for name, x in (("o", O), ("lse", lse), ("dk", dK), ("dv", dV), ("dtable", dT)):
        if x is not None:
            _check(x, val, err, name)
    got, want = _host(dQ), val["dq"]
    fits = np.abs(want).max(3) < 65504                     # some large rows go beyond fp16's largest number
    assert fits[:, 1::2].all()
    off, size = (np.linalg.norm(x, axis=3) for x in (np.where(fits[..., None], got - want, 0), want))
    assert size[:, 1::2].min() > 2.0 ** -10                # eight normal features of 2^-14 and more: no steps of subnormal results
    assert np.all(off <= 3 * A.UNIT["f16"] * size)


@pytest.mark.parametrize("edges", [None, EDGES])
@pytest.mark.parametrize("what", ["batch", "heads"])
@pytest.mark.parametrize("name", ["dq", "dk"])
def test_small_gradients_of_a_batch_beside_large_ones_in_fp16(ctx, edges, what, name):
    """dO and V at 2^5 in one half of the batch (or of the shared heads) and at 2^-5 in the other: they meet in no sum of dQ and dK, so each half is as
    precise as alone.  In the 2-norm one u each for a rounding of dS, of delta's o and of the result.  (The scale of 64 that lifts a result
    out of the subnormal numbers is taken back in the other operand.)"""
    rng = np.random.default_rng(40)
    att, dO = _case(rng, "f16", 2, 4, 2, 120, 2000, 64, 64, edges=edges)
    att.scale = 64.0
    (att.Q if name == "dq" else att.K).mul_(2.0 ** -9)
    size = torch.tensor([2.0 ** 5, 2.0 ** -5], device=DEV, dtype=torch.float16)
    if what == "batch":
        att.V.mul_(size[:, None, None, None])
        dO.mul_(size[:, None, None, None])
    else:
        att.V.mul_(size[:, None])
        dO.mul_(size.repeat_interleave(2)[:, None])
    val, _ = _oracle("f16", att, dO)
    O, lse = ctx.bbmm_attend(att)
    grads = ctx.bbmm_attend_grad(att, O, lse, dO)
    got, want = _host(grads[0 if name == "dq" else 1]), val[name]
    half = want.shape[2] // 2
    got, want = (x[1] if what == "batch" else x[:, :, half:] for x in (got, want))
    assert np.linalg.norm(want) > 2.0 ** -12 * np.sqrt(want.size)      # normal numbers
    assert np.linalg.norm(got - want) <= 3 * A.UNIT["f16"] * np.linalg.norm(want)


def test_lengths_do_not_change_the_parts_of_fp32(ctx):
    """Finer parts of a split key axis even out unequal lengths, but cost fp32 more than that: a batch with lengths is split as one without."""
    from paper_1809_11165_amd import binding
    q = torch.zeros(8, 1, 32, 128, device=DEV)
    kv = torch.zeros(1, 1, 8, 128, device=DEV).expand(8, 32773, 8, 128)
    k_len = torch.full((8,), 32773, dtype=torch.int32, device=DEV)
    plain, full = binding.Attention(q, kv, kv), binding.Attention(q, kv, kv, k_len=k_len)
    assert ctx.bbmm_attend_workspace(plain) == ctx.bbmm_attend_workspace(full) > 0


def test_inputs_that_require_grad_are_refused(ctx):
    """No call is part of a recorded graph of gradients: inputs that such a graph is to follow are refused rather than left out of it."""
    att, dO = _case(np.random.default_rng(41), "f32", 1, 2, 2, 5, 9, 16, 16, edges=EDGES)
    O, lse = ctx.bbmm_attend(att)
    want = ctx.bbmm_attend_grad(att, O, lse, dO)
    for name in ("Q", "K", "V", "table"):
        leaf = getattr(att, name).requires_grad_()
        for call in (lambda: ctx.bbmm_attend(att), lambda: ctx.bbmm_attend_grad(att, O, lse, dO)):
            with pytest.raises(ValueError, match="requires? grad"):
                call()
        with torch.no_grad():
            assert torch.equal(ctx.bbmm_attend(att)[0], O)
            assert all(torch.equal(x, y) for x, y in zip(ctx.bbmm_attend_grad(att, O, lse, dO), want))
        leaf.requires_grad_(False)
    table = att.table.requires_grad_()
    with pytest.raises(ValueError):
        ctx.bbmm_bucket_bias(table, EDGES, 4, 4)
    dB = torch.zeros(1, 2, 4, 4, device=DEV, requires_grad=True)
    with pytest.raises(ValueError):
        ctx.bbmm_bucket_bias_grad(dB, EDGES)
    with torch.no_grad():
        assert ctx.bbmm_bucket_bias(table, EDGES, 4, 4).shape == (2, 4, 4)


def test_the_calls_inside_a_function_of_torch(ctx):
    """As a model uses them: the calls as forward and backward of an autograd function, whose gradients are those of the call."""
    from paper_1809_11165_amd import binding

    class Read(torch.autograd.Function):
        @staticmethod
        def forward(save, Q, K, V, table):
            att = binding.Attention(Q, K, V, table=table, edges=EDGES)
            O, lse = ctx.bbmm_attend(att)
            save.att = att
            save.save_for_backward(O, lse)
            return O

        @staticmethod
        def backward(save, dO):
            return ctx.bbmm_attend_grad(save.att, *save.saved_tensors, dO)

    att, dO = _case(np.random.default_rng(42), "f32", 2, 4, 2, 40, 70, 32, 32, edges=EDGES)
    O, lse = ctx.bbmm_attend(att)
    want = ctx.bbmm_attend_grad(att, O, lse, dO)
    leaves = [x.clone().requires_grad_() for x in (att.Q, att.K, att.V, att.table)]
    (Read.apply(*leaves) * dO).sum().backward()
    torch.cuda.synchronize()
    for leaf, x in zip(leaves, want):
        assert torch.equal(leaf.grad, x)


# batch times kv_heads a multiple of eight: units of several workgroups dealt out to the dies one by one, in all three kernels
DEALT = {
    "units_8": (4, 4, 2, 150, 200, 64, 64, dict(edges=EDGES)),
    "units_16_ragged": (8, 4, 2, 300, 333, 40, 40, dict(edges=EDGES, k_len=[333, 0, 1, 200, 150, 333, 64, 129], q_len=[300, 300, 5, 0, 128, 129, 300, 1])),
    "units_8_split": (2, 4, 4, 140, 1500, 64, 64, dict(edges=EDGES, start=[1300, -20], mask=0.8)),
    "units_8_wide": (1, 16, 8, 260, 300, 128, 128, {}),
}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(DEALT))
def test_units_dealt_out_over_the_dies(ctx, name, kind):
    *shape, opt = DEALT[name]
    att, dO = _case(np.random.default_rng(sum(map(ord, name))), kind, *shape, **opt)
    _run_and_check(ctx, kind, att, dO)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [4, 70])
def test_a_causal_table_beside_a_head_of_the_lowest_value(ctx, kind, nq):
    """The head of the causal table, element by element, in every type; the other head's bias flattens its rows."""
    rng = np.random.default_rng(38)
    att, dO = _case(rng, kind, 1, 2, 2, nq, 40, 32, 32, edges=EDGES, start=[-3])
    n = len(EDGES) + 1
    att.table[0, n:] = -float("inf")
    att.table[0, 0] = -float("inf")
    att.table[1, :] = torch.finfo(TYPES[kind]).min
    val, err = _oracle(kind, att, dO)
    O, lse = ctx.bbmm_attend(att)
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    assert all(torch.isfinite(x).all() for x in (O, dQ, dK, dV, dT))
    _check(lse[:, :1], {"lse": val["lse"][:, :1]}, {"lse": err["lse"][:, :1]}, "lse")
    for name, x in (("o", O), ("dq", dQ), ("dk", dK), ("dv", dV)):
        _check(x[:, :, :1], {name: val[name][:, :, :1]}, {name: err[name][:, :, :1]}, name)
    _check(dT[:1], {"dtable": val["dtable"][:1]}, {"dtable": err["dtable"][:1]}, "dtable")


def _f32_gradients(att, dO, dtype):
    """The formula by elementary products in `dtype`, on the GPU: dq, dk, dv and dtable."""
    B, nq, H, d = att.Q.shape
    nk, HK = att.K.shape[1:3]
    G, edges = H // HK, att.edges
    q, do = (x.to(dtype).transpose(1, 2).contiguous() for x in (att.Q, dO))
    k, v = (x.to(dtype).transpose(1, 2).repeat_interleave(G, 1).contiguous() for x in (att.K, att.V))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5
    n = None
    if att.table is not None:
        r = torch.arange(nk, device=DEV)[None, :] - torch.arange(nq, device=DEV)[:, None]
        n = torch.from_numpy(A.bucket(r.cpu().numpy(), edges, att.two_sided)).to(DEV)
        s = s + att.table.to(dtype)[:, n]
    p = torch.exp(s - s.amax(3, keepdim=True))
    p = p / p.sum(3, keepdim=True)
    o = torch.matmul(p, v)
    ds = p * (torch.matmul(do, v.transpose(2, 3).contiguous()) - (do * o).sum(3, keepdim=True))
    out = {"dq": (torch.matmul(ds, k) * d ** -0.5).transpose(1, 2)}
    for name, x, y in (("dk", ds * d ** -0.5, q), ("dv", p, do)):
        z = torch.matmul(x.transpose(2, 3).contiguous(), y)
        out[name] = z.view(B, HK, G, nk, -1).sum(2).transpose(1, 2)
    if n is not None:
        rows = ds.double().sum(0).reshape(H, -1)
        out["dtable"] = torch.zeros(H, att.table.shape[1], device=DEV, dtype=torch.float64).index_add_(1, n.reshape(-1), rows).to(dtype)
    return out


@pytest.mark.parametrize("B,H,HK,nq,nk,d,dv,edges,two_sided", [
    (2, 1, 1, 2627, 484, 96, 16, [1, 2, 3, 4, 5, 7, 10, 14, 20, 30, 42], True),
    (3, 1, 1, 2249, 998, 80, 80, list(range(1, 17)) + [20, 26, 33, 43, 55], False),
    (4, 1, 1, 407, 5859, 16, 64, [1, 2, 5, 12, 20], True),
    (4, 2, 2, 1509, 2854, 32, 16, None, True),
    (3, 2, 2, 2612, 86, 32, 32, [1, 2, 40], True),          # nearly all rows beyond the last edge
    (2, 6, 3, 300, 300, 128, 128, [1, 1000], True),         # and all of them between two
    (1, 8, 1, 150, 3000, 40, 40, EDGES, True),              # parts of both axes, many heads a workgroup
])
def test_fp32_gradients_are_as_precise_as_the_formula_in_fp32(ctx, B, H, HK, nq, nk, d, dv, edges, two_sided):
    """Against 64 bits the 2-norm of a gradient's error is at most one and a half times that of the formula's own steps in fp32, or 4 u32: root mean
    squares over four inputs, as a bucket that holds most of all rows is one number, in which either side's rounding may happen to cancel."""
    off, of_plain = {}, {}
    for seed in range(4):
        att, dO = _case(np.random.default_rng(seed), "f32", B, H, HK, nq, nk, d, dv, edges=edges, two_sided=two_sided)
        exact, plain = (_f32_gradients(att, dO, t) for t in (torch.float64, torch.float32))
        O, lse = ctx.bbmm_attend(att)
        for name, x in zip(("dq", "dk", "dv", "dtable"), ctx.bbmm_attend_grad(att, O, lse, dO)):
            for sums, y in (off, x), (of_plain, plain.get(name)):
                if x is not None:
                    sums[name] = sums.get(name, 0.0) + float((y.double() - exact[name]).norm() / exact[name].norm()) ** 2 / 4
    for name in off:
        assert off[name] ** 0.5 <= max(1.5 * of_plain[name] ** 0.5, 4 * A.U32), (name, off[name] ** 0.5, of_plain[name] ** 0.5)
