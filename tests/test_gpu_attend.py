"""GPU parity of the attention entry points, forward and gradient, through the C ABI: every element against the fp64 oracle within the
rounding bounds that oracle/attend_oracle.py derives, over types, head sharing, odd sizes, empty rows and axes, lengths, masks, strides,
garbage in places that take no part, split key axes, streams and graphs."""
import numpy as np
import pytest

from oracle import attend_oracle as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_1809_11165_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


def _rand(rng, kind, *shape, spread=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * spread).astype(np.float32)).to(DEV).to(TYPES[kind])


def _host(x):
    return None if x is None else x.detach().to("cpu").to(torch.float64).numpy()


def _check(got, val, err, name):
    g = _host(got)
    assert g.shape == val[name].shape, name
    finite = np.isfinite(val[name])
    assert np.array_equal(g[~finite], val[name][~finite]), name
    assert np.all(np.isfinite(g[finite])), name
    off = np.abs(g[finite] - val[name][finite])
    lim = err[name][finite]
    bad = off > lim
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its bound" % (name, bad.sum(), bad.size, (off[bad] / np.maximum(lim[bad], 1e-300)).max())


def _case(rng, kind, B, H, HK, nq, nk, d, dv, edges=None, two_sided=True, start=None, q_len=None, k_len=None, mask=None):
    from paper_1809_11165_amd import binding
    t = {"Q": _rand(rng, kind, B, nq, H, d), "K": _rand(rng, kind, B, nk, HK, d), "V": _rand(rng, kind, B, nk, HK, dv)}
    kw = {}
    if edges is not None:
        kw["table"] = _rand(rng, kind, H, (len(edges) + 1) * (2 if two_sided else 1))
        kw["edges"], kw["two_sided"] = edges, two_sided
        if start is not None:
            kw["q_start"] = torch.tensor(start, dtype=torch.int64, device=DEV)
    if q_len is not None:
        kw["q_len"] = torch.tensor(q_len, dtype=torch.int32, device=DEV)
    if k_len is not None:
        kw["k_len"] = torch.tensor(k_len, dtype=torch.int32, device=DEV)
    if mask is not None:
        kw["key_mask"] = torch.from_numpy(rng.random((B, nk)) < mask).to(DEV)
    return binding.Attention(t["Q"], t["K"], t["V"], **kw), _rand(rng, kind, B, nq, H, dv)


def _oracle(kind, att, dO=None):
    scale = att.Q.shape[3] ** -0.5 if att.scale is None else att.scale
    return A.attend(kind, _host(att.Q), _host(att.K), _host(att.V), scale, dO=_host(dO), q_len=_host(att.q_len), k_len=_host(att.k_len),
                    mask=_host(att.key_mask), table=_host(att.table), edges=att.edges or (), two_sided=att.two_sided, start=_host(att.q_start))


def _run_and_check(ctx, kind, att, dO, oracle=None):
    val, err = oracle or _oracle(kind, att, dO)
    O, lse = ctx.bbmm_attend(att)
    _check(O, val, err, "o")
    _check(lse, val, err, "lse")
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    for name, x in (("dq", dQ), ("dk", dK), ("dv", dV), ("dtable", dT)):
        if x is not None:
            _check(x, val, err, name)
    assert (dT is None) == (att.table is None)
    return O, lse, dQ, dK, dV, dT


EDGES = [1, 2, 3, 4, 6, 9, 14, 21]

# B, H, HK, nq, nk, d, dv, options
CASES = {
    "one_query_one_key": (1, 1, 1, 1, 1, 64, 64, {}),
    "one_query": (2, 4, 4, 1, 77, 64, 64, dict(edges=EDGES)),
    "one_query_shared_split": (2, 8, 2, 1, 2500, 128, 128, dict(k_len=[2500, 1301])),
    "few_rows_shared_bias_split": (1, 6, 2, 7, 1500, 40, 40, dict(edges=EDGES, start=[1493])),
    "few_rows_start_far_behind": (2, 2, 1, 3, 90, 24, 24, dict(edges=EDGES, start=[-(1 << 50), 1 << 50])),
    "one_key": (2, 2, 2, 70, 1, 32, 32, dict(edges=EDGES)),
    "tile_exact": (1, 2, 2, 128, 64, 64, 64, {}),
    "tile_plus_one": (1, 2, 2, 129, 65, 64, 64, dict(edges=EDGES)),
    "odd": (2, 3, 1, 201, 157, 33, 7, dict(edges=EDGES, start=[5, -40], k_len=[157, 90], q_len=[201, 33])),
    "odd_one_sided": (1, 4, 4, 150, 333, 20, 20, dict(edges=EDGES, two_sided=False, start=[200])),
    "wide_features": (1, 2, 1, 140, 260, 128, 128, dict(edges=EDGES, mask=0.8)),
    "values_wider": (1, 2, 2, 65, 100, 16, 128, {}),
    "one_feature": (1, 2, 2, 40, 50, 1, 1, {}),
    "no_edges": (1, 2, 2, 45, 70, 64, 64, dict(edges=[])),
    "far_edges": (1, 1, 1, 200, 1400, 64, 64, dict(edges=[1, 100, 700, 1024], start=[300])),
    "far_edges_wide": (1, 2, 1, 150, 300, 128, 100, dict(edges=[3, 400, 1024], start=[80])),
    "many_heads_one_query": (2, 100, 1, 1, 400, 64, 64, dict(edges=EDGES, start=[399, 200])),
    "wide_group": (1, 24, 2, 33, 300, 40, 40, dict(edges=EDGES)),
    "empty_batches": (3, 2, 2, 50, 60, 64, 64, dict(k_len=[0, 60, 1], q_len=[50, 0, 50], edges=EDGES)),
    "empty_batches_few": (3, 2, 2, 2, 300, 64, 64, dict(k_len=[0, 300, 1], q_len=[2, 0, 1], edges=EDGES)),
    "split_rows": (1, 1, 1, 90, 2100, 64, 64, dict(edges=EDGES, start=[2000], k_len=[2050])),
    "sparse_mask": (2, 2, 2, 60, 400, 64, 64, dict(mask=0.03)),
    "lengths_out_of_range": (2, 2, 2, 40, 50, 64, 64, dict(k_len=[-3, 1000], q_len=[1000, -1])),
}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(CASES))
def test_forward_and_gradients_match_the_oracle(ctx, name, kind):
    *shape, opt = CASES[name]
    att, dO = _case(np.random.default_rng(sum(map(ord, name))), kind, *shape, **opt)
    _run_and_check(ctx, kind, att, dO)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [2, 100])
def test_rows_that_a_mask_empties_and_garbage_in_masked_places(ctx, kind, nq):
    rng = np.random.default_rng(5)
    att, dO = _case(rng, kind, 2, 2, 1, nq, 130, 64, 64, edges=EDGES, k_len=[100, 130], q_len=[nq, nq - 1], mask=0.7)
    att.key_mask[1] = False                                # a batch that its mask leaves nothing of
    want = _oracle(kind, att, dO)
    gone = ~(att.key_mask & (torch.arange(130, device=DEV)[None] < att.k_len[:, None]))
    for x, bad in ((att.K, float("nan")), (att.V, float("inf"))):
        x[gone] = bad
    att.V[0, 129] = float("nan")
    att.Q[1, nq - 1], dO[1, nq - 1] = float("nan"), float("inf")
    O, lse, dQ, dK, dV, dT = _run_and_check(ctx, kind, att, dO, want)
    assert torch.all(O[1] == 0) and torch.all(lse[1] == -float("inf")) and torch.all(dQ[1] == 0)
    assert torch.all(dK[gone] == 0) and torch.all(dV[gone] == 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [2, 100])
def test_signalling_nan_in_masked_places(ctx, kind, nq):
    rng = np.random.default_rng(18)
    att, dO = _case(rng, kind, 2, 2, 1, nq, 130, 64, 64, edges=EDGES, mask=0.7)
    want = _oracle(kind, att, dO)
    bits = {"f32": (torch.int32, 0x7f800001), "f16": (torch.int16, 0x7c01), "bf16": (torch.int16, 0x7f81)}[kind]
    for x in (att.K, att.V):
        x.view(bits[0])[~att.key_mask] = bits[1]
    _run_and_check(ctx, kind, att, dO, want)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [4, 70])
def test_tables_of_minus_infinity_and_of_the_lowest_value(ctx, kind, nq):
    """-infinity for everything ahead (a causal mask by the table), and buckets at the type's lowest value: weight zero beside any other
    score, equal weights where a row holds nothing else."""
    rng = np.random.default_rng(6)
    att, dO = _case(rng, kind, 1, 2, 2, nq, 40, 32, 32, edges=EDGES, start=[-3])
    n = len(EDGES) + 1
    att.table[0, n:] = -float("inf")                       # keys ahead of the query
    att.table[0, 0] = -float("inf")                        # and its own: early rows keep nothing
    att.table[1, :] = torch.finfo(TYPES[kind]).min
    if kind == "f32":
        att.table[1, :] = -2.2e38                          # see the note on entries below -2.3e38
    val, err = _oracle(kind, att, dO)
    if kind != "f16":                                      # beside it a score of the usual size is rounded away: equal weights
        keys = _host(att.V)[0, :, 1]
        val["o"][0, :, 1] = keys.mean(0)
        O, lse = ctx.bbmm_attend(att)
        u = A.UNIT[kind]
        assert np.all(np.abs(_host(O)[0, :, 1] - keys.mean(0)) <= (2 * u + 64 * A.U32) * np.abs(keys).mean(0))
        assert torch.isfinite(lse[:, 1]).all()
        return
    O, lse = ctx.bbmm_attend(att)
    assert torch.isfinite(O).all()
    _check(lse[:, :1], {"lse": val["lse"][:, :1]}, {"lse": err["lse"][:, :1]}, "lse")
    _check(O[:, :, :1], {"o": val["o"][:, :, :1]}, {"o": err["o"][:, :, :1]}, "o")


@pytest.mark.parametrize("kind,value", [("f32", -3.4028234663852886e38), ("f32", -1e9), ("bf16", -3.3895313892515355e38), ("bf16", -1e9), ("f32", 1e9)])
@pytest.mark.parametrize("nq", [4, 70])
@pytest.mark.parametrize("edges", [EDGES, [1]])
def test_gradients_of_rows_that_a_huge_bias_flattens(ctx, kind, value, nq, edges):
    """A bias that rounds every score away leaves equal weights: o and dv are means, dS = (dP - delta) / n, and none of it recoverable from an
    fp32 lse.  Scores are kept below the rounding of 1e9 (64), so that they vanish in it."""
    rng = np.random.default_rng(17)
    att, dO = _case(rng, kind, 2, 2, 1, nq, 200, 32, 32, edges=edges, k_len=[200, 131])
    att.table[:] = value
    flat = type(att)(att.Q, att.K, att.V, scale=1e-30, k_len=att.k_len)
    val, err = _oracle(kind, flat, dO)                     # weights 1 / n; dq and dk carry the scale
    O, lse = ctx.bbmm_attend(att)
    _check(O, val, err, "o")
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    _check(dV, val, err, "dv")
    factor = 32 ** -0.5 / 1e-30
    tiny = {"dq": 0.0, "dk": 0.0}
    for name, x in (("dq", dQ), ("dk", dK)):
        _check(x, {name: val[name] * factor}, {name: err[name] * factor + tiny[name]}, name)
    with_table = A.attend(kind, _host(att.Q), _host(att.K), _host(att.V), 1e-30, dO=_host(dO), k_len=_host(att.k_len),
                          table=np.zeros(tuple(att.table.shape)), edges=edges)
    _check(dT, with_table[0], with_table[1], "dtable")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq", [4, 70])
def test_a_causal_table_has_gradients(ctx, kind, nq):
    rng = np.random.default_rng(7)
    att, dO = _case(rng, kind, 1, 2, 2, nq, 90, 32, 32, edges=EDGES, start=[-3])
    att.table[:, len(EDGES) + 1:] = -float("inf")
    val, err = _oracle(kind, att, dO)
    assert np.isinf(val["lse"][0, 0, 3:]).sum() == 0 and np.isinf(val["lse"][0, 0, :3]).all()
    _, _, _, _, _, dT = _run_and_check(ctx, kind, att, dO, (val, err))
    assert torch.all(dT[:, len(EDGES) + 1:] == 0)


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_orders_and_alignment(ctx, kind):
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(8)
    B, H, HK, nq, nk, d = 2, 4, 2, 75, 140, 32
    base, dO = _case(rng, kind, B, H, HK, nq, nk, d, d, edges=EDGES)
    want = _oracle(kind, base, dO)
    got = [ctx.bbmm_attend(base)]
    got[0] += ctx.bbmm_attend_grad(base, *got[0], dO)

    def heads_first(x):                                    # (batch, head, row, feature) in memory
        return x.transpose(1, 2).contiguous().transpose(1, 2)

    def in_wider_rows(x, lead):                            # a slice of wider rows; lead 1: not aligned to 16 bytes
        y = torch.full((*x.shape[:3], x.shape[3] + 9), float("nan"), dtype=x.dtype, device=DEV)
        y[..., lead:lead + x.shape[3]] = x
        return y[..., lead:lead + x.shape[3]]

    for change in (heads_first, lambda x: in_wider_rows(x, 0), lambda x: in_wider_rows(x, 1)):
        att = binding.Attention(change(base.Q), change(base.K), change(base.V), table=base.table, edges=EDGES)
        _run_and_check(ctx, kind, att, change(dO), want)
        O, lse = ctx.bbmm_attend(att)
        for x, y in zip((O, lse) + ctx.bbmm_attend_grad(att, O, lse, change(dO)), got[0]):
            assert torch.equal(x, y)                       # the same numbers whatever the layout
    # a key axis shared by the batch: stride zero, a gradient for every use
    shared = binding.Attention(base.Q, base.K[:1].expand(B, -1, -1, -1), base.V[:1].expand(B, -1, -1, -1), table=base.table, edges=EDGES)
    _run_and_check(ctx, kind, shared, dO)


def test_an_offset_beyond_32_bits(ctx):
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(9)
    nk, d, stride = 300, 32, 9_000_000                     # the last row starts 2.7e9 elements in
    room = torch.empty(nk * stride, dtype=torch.bfloat16, device=DEV)
    K = room.as_strided((1, nk, 1, d), (0, stride, d, 1))
    V = room.as_strided((1, nk, 1, d), (0, stride, d, 1), 64)
    K.copy_(_rand(rng, "bf16", 1, nk, 1, d))
    V.copy_(_rand(rng, "bf16", 1, nk, 1, d))
    for nq in (3, 70):
        att = binding.Attention(_rand(rng, "bf16", 1, nq, 1, d), K, V)
        _run_and_check(ctx, "bf16", att, _rand(rng, "bf16", 1, nq, 1, d))
    del room


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("sizes", [(0, 2, 5, 7), (2, 2, 0, 7), (2, 2, 5, 0), (1, 2, 200, 0)])
def test_axes_of_no_length(ctx, kind, sizes):
    B, H, nq, nk = sizes
    att, dO = _case(np.random.default_rng(10), kind, B, H, H, nq, nk, 16, 16, edges=EDGES)
    O, lse = ctx.bbmm_attend(att)
    assert O.shape == (B, nq, H, 16) and torch.all(O == 0) and torch.all(lse == -float("inf"))
    for x in ctx.bbmm_attend_grad(att, O, lse, dO):
        assert torch.all(x == 0)


def test_small_gradients_and_long_rows_in_fp16(ctx):
    """Weights of 1 / 6000 and gradients of 1e-4: both would be subnormal in fp16 without scaling."""
    rng = np.random.default_rng(11)
    att, dO = _case(rng, "f16", 1, 1, 1, 64, 6000, 32, 32, edges=EDGES)
    att.Q.mul_(0.1)
    dO.mul_(1e-4)
    val, err = _oracle("f16", att, dO)
    O, lse, dQ, dK, dV, dT = _run_and_check(ctx, "f16", att, dO, (val, err))
    for name, x in (("dq", dQ), ("dv", dV)):
        # outputs of 1e-6 and below are steps of fp16 themselves (2^-24): compare with the rounded value
        ref = torch.from_numpy(val[name]).to(torch.float16).double().numpy()
        assert np.abs(_host(x) - ref).max() <= 2 * 2.0 ** -24


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("nk", [1, 3, 8, 33, 100, 250])
def test_short_rows_keep_the_precision_of_their_type(ctx, kind, nk):
    """delta from the rounded o would cost rows of few keys several roundings in the table's gradient.  With delta from the scores the gradients
    are off by one rounding of the output and (dQ, dK) one of dS each: 2 roundings of u in the 2-norm bound any mix of them, and 64 u32 the
    fp32 sums."""
    rng = np.random.default_rng(19)
    att, dO = _case(rng, kind, 2, 4, 2, 300, nk, 64, 64, edges=EDGES, start=[-nk, nk // 2])
    val, _ = _oracle(kind, att, dO)
    O, lse = ctx.bbmm_attend(att)
    dQ, dK, dV, dT = ctx.bbmm_attend_grad(att, O, lse, dO)
    u = A.UNIT[kind]
    for name, x, units in (("dq", dQ, 2), ("dk", dK, 2), ("dv", dV, 2), ("dtable", dT, 1)):
        size = np.linalg.norm(val[name])
        if nk > 1 or name == "dv":                         # one key: weights one, dS zero
            assert np.linalg.norm(_host(x) - val[name]) <= (units * u + 64 * A.U32) * size, name
        else:
            assert np.abs(_host(x)).max() <= 64 * A.U32 * 300 * 64


@pytest.mark.parametrize("nq,nk", [(3, 700), (150, 700)])
def test_gradients_against_differences(ctx, nq, nk):
    """sum(dO . O) along a random direction of all inputs together, fp32: central differences of step 2^-6 differ from the derivative by
    h^2 / 6 times a third derivative of order one, and by rounding of about 1e-6 / h."""
    rng = np.random.default_rng(12)
    att, dO = _case(rng, "f32", 2, 4, 2, nq, nk, 32, 32, edges=EDGES, mask=0.9, start=[0, 40])
    O, lse = ctx.bbmm_attend(att)
    grads = ctx.bbmm_attend_grad(att, O, lse, dO)
    inputs = (att.Q, att.K, att.V, att.table)
    for which in range(4):
        step = torch.from_numpy(rng.standard_normal(tuple(inputs[which].shape)).astype(np.float32)).to(DEV)
        want = float((grads[which].double() * step.double()).sum())
        at, h = [], 2.0 ** -6
        for sign in (1, -1):
            keep = inputs[which].clone()
            inputs[which].add_(step, alpha=sign * h)
            at.append(float((ctx.bbmm_attend(att)[0].double() * dO.double()).sum()))
            inputs[which].copy_(keep)
        got = (at[0] - at[1]) / (2 * h)
        size = float((grads[which].double() ** 2).sum()) ** 0.5
        assert abs(got - want) <= 2e-2 * size, (which, got, want, size)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("nq,nk", [(1, 3500), (300, 500)])
def test_the_same_call_gives_the_same_bits(ctx, kind, nq, nk):
    att, dO = _case(np.random.default_rng(13), kind, 2, 4, 2, nq, nk, 64, 64, edges=EDGES)
    first = ctx.bbmm_attend(att)
    first += ctx.bbmm_attend_grad(att, *first, dO)
    for _ in range(3):
        again = ctx.bbmm_attend(att)
        again += ctx.bbmm_attend_grad(att, *again, dO)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_streams_of_the_context_and_of_the_caller(ctx):
    """A context on a stream of its own, called with inputs that the caller's stream is still writing, and results used there."""
    from paper_1809_11165_amd import binding
    att, dO = _case(np.random.default_rng(14), "bf16", 2, 4, 4, 200, 900, 64, 64, edges=EDGES)
    want = ctx.bbmm_attend(att)
    want += ctx.bbmm_attend_grad(att, *want, dO)
    torch.cuda.synchronize()
    other = binding.Context(0, stream=torch.cuda.Stream())
    try:
        for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
            with torch.cuda.stream(stream):
                late = torch.empty_like(att.Q)
                torch.cuda._sleep(2_000_000)
                late.copy_(att.Q)
                a = binding.Attention(late, att.K, att.V, table=att.table, edges=EDGES)
                O, lse = other.bbmm_attend(a)
                got = (O, lse) + other.bbmm_attend_grad(a, O, lse, dO)
                copies = [x.clone() for x in got]
                del late, a, got, O, lse
            stream.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(copies, want))
    finally:
        other.close()


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_two_recorded_training_steps_replayed_in_turn(kind):
    """Two graphs from one context, of different sizes: their workspaces come from the recording's own memory, so neither spoils the
    other, nor does eager work between the replays."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(15)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        cases = [_case(rng, kind, 2, 4, 2, 1, 3000, 64, 64, edges=EDGES), _case(rng, kind, 1, 4, 4, 150, 260, 64, 64, edges=EDGES)]

        def step(att, dO):
            O, lse = ctx.bbmm_attend(att)
            return (O, lse) + ctx.bbmm_attend_grad(att, O, lse, dO)

        for c in cases:
            step(*c)
        stream.synchronize()
        graphs = []
        for c in cases:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = step(*c)
            graphs.append((g, out))
        for turn in range(3):
            for c in cases:
                c[0].Q.copy_(_rand(rng, kind, *c[0].Q.shape))
                c[1].copy_(_rand(rng, kind, *c[1].shape))
            for g, _ in graphs:
                g.replay()
            eager = [step(*c) for c in cases]
            stream.synchronize()
            for (_, out), e in zip(graphs, eager):
                assert all(torch.equal(x, y) for x, y in zip(out, e)), turn
        del graphs
    ctx.close()


def test_refusals_of_the_library(ctx):
    import ctypes as C
    from paper_1809_11165_amd import binding
    att, dO = _case(np.random.default_rng(16), "f32", 1, 4, 2, 40, 50, 16, 16, edges=EDGES)
    O, lse = ctx.bbmm_attend(att)

    def refused(change, needle, att=att):
        a = att.to_c(ctx.device)
        change(a)
        rc = ctx.lib.bbmm_attend(ctx.h, C.byref(a), binding._dptr(O), binding._dptr(lse), None, 0)
        assert rc == binding.EINVAL and needle in ctx.lib.bbmm_last_error(ctx.h).decode()

    def put(name, value):
        return lambda a: setattr(a, name, value)

    refused(put("type", 7), "type")
    refused(put("kv_heads", 3), "kv_heads")
    refused(put("kv_heads", 0), "kv_heads")
    refused(put("batch", -1), "batch")
    refused(put("nq", -1), "nq")
    refused(put("nk", (1 << 30) + 1), "nk")
    refused(put("d", 129), "d and dv")
    refused(put("dv", 0), "d and dv")
    for s in (0.0, -1.0, float("inf"), float("nan"), 1e-60):
        refused(put("scale", s), "scale")
    refused(put("Q", None), "required")
    refused(put("V", None), "required")
    refused(put("K", att.K.data_ptr() + 2), "aligned")
    refused(lambda a: a.q_stride.__setitem__(1, -16), "stride")
    refused(put("n_edges", 64), "edges")
    refused(put("edges", None), "edges")
    for bad in ([0, 1], [1, 1], [3, 2], [1, 1025]):
        e = (C.c_int32 * 2)(*bad)
        def edges(a, e=e):
            a.n_edges, a.edges = 2, e
        refused(edges, "edges")
    a = att.to_c(ctx.device)
    assert ctx.lib.bbmm_attend(ctx.h, C.byref(a), None, binding._dptr(lse), None, 0) == binding.EINVAL
    assert ctx.lib.bbmm_attend(ctx.h, None, binding._dptr(O), binding._dptr(lse), None, 0) == binding.EINVAL
    assert ctx.lib.bbmm_attend(None, C.byref(a), binding._dptr(O), binding._dptr(lse), None, 0) == binding.EINVAL
    with pytest.raises(binding.BbmmError):                  # more rows than a launch takes
        many = binding.Attention(att.Q.expand(1, 40, 4, 16), att.K, att.V)
        b = many.to_c(ctx.device)
        b.nq = 1 << 30
        ctx._attend_bytes(b, True)
    # workspaces: too small, missing, not aligned
    need = ctx.bbmm_attend_workspace(att, grad=True)
    room = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
    stride = (C.c_int64 * 3)(*dO.stride()[:3])
    g = [torch.empty_like(x) for x in (att.Q, att.K, att.V, att.table)]
    for ptr, n in ((room.data_ptr(), need - 1), (None, need), (room.data_ptr() + 4, need)):
        rc = ctx.lib.bbmm_attend_grad(ctx.h, C.byref(a), binding._dptr(O), binding._dptr(lse), binding._dptr(dO), stride,
                                      *[binding._dptr(x) for x in g], ptr, n)
        assert rc == binding.EINVAL and "workspace" in ctx.lib.bbmm_last_error(ctx.h).decode()
    rc = ctx.lib.bbmm_attend_grad(ctx.h, C.byref(a), binding._dptr(O), binding._dptr(lse), binding._dptr(dO), stride,
                                  *[binding._dptr(x) for x in g[:3]], None, room.data_ptr(), need)
    assert rc == binding.EINVAL and "dtable" in ctx.lib.bbmm_last_error(ctx.h).decode()
    # the context still works
    again = ctx.bbmm_attend(att)
    assert torch.equal(again[0], O) and torch.equal(again[1], lse)


def test_refusals_of_scales_lengths_and_starts(ctx):
    import ctypes as C
    from paper_1809_11165_amd import binding
    att, dO = _case(np.random.default_rng(21), "f32", 2, 2, 2, 5, 9, 16, 16)
    O, lse = ctx.bbmm_attend(att)
    for change in (dict(scale=3e38), dict(q_len=2), dict(k_len=1), dict(q_start=4)):      # the last three: addresses off by that much
        a = att.to_c(ctx.device)
        for name, x in change.items():
            setattr(a, name, x if name == "scale" else O.data_ptr() + x)
        rc = ctx.lib.bbmm_attend(ctx.h, C.byref(a), binding._dptr(O), binding._dptr(lse), None, 0)
        assert rc == binding.EINVAL, change
    none = binding.Attention(att.Q[..., :0], att.K[..., :0], att.V)
    with pytest.raises(binding.BbmmError) as e:
        ctx.bbmm_attend(none)
    assert e.value.code == binding.EINVAL


def test_two_contexts_at_work_at_once():
    """Each on a stream of its own, their calls queued in turn without a wait between: the results are those of a context alone."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(22)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [binding.Context(0, stream=s) for s in streams]
    cases = [_case(rng, "f16", 2, 4, 2, 300, 700, 64, 64, edges=EDGES), _case(rng, "bf16", 2, 8, 2, 1, 5000, 128, 128, edges=EDGES)]

    def step(k):
        with torch.cuda.stream(streams[k]):
            O, lse = ctxs[k].bbmm_attend(cases[k][0])
            return (O, lse) + ctxs[k].bbmm_attend_grad(cases[k][0], O, lse, cases[k][1])

    torch.cuda.synchronize()
    want = []
    for k in (0, 1):
        want.append(step(k))
        torch.cuda.synchronize()
    got = [[step(k) for k in (0, 1)] for _ in range(10)]
    torch.cuda.synchronize()
    for pair in got:
        for k in (0, 1):
            assert all(torch.equal(x, y) for x, y in zip(pair[k], want[k]))
    for c in ctxs:
        c.close()


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("nq,nk,edges,two_sided,start", [
    (37, 2171, [1, 3, 12], True, 2134),           # nearly all of a row behind the last edge; keys split over workgroups
    (741, 1498, [1, 2, 3, 4, 5, 8, 13, 28], False, 0),    # and all of many rows in one bucket
    (1281, 333, [1, 13, 170], True, 0),
    (90, 900, [1, 1000], True, 40),               # in one between two edges
    (5, 9000, EDGES, True, 8990),
])
def test_a_table_of_rows_that_lie_in_one_bucket(ctx, kind, nq, nk, edges, two_sided, start):
    """A row's dS sum to zero, so little is left of a bucket that holds nearly all of it: the rounding of o must not stand there.  Bound:
    half a step of the result, and 64 u32 of what the sums are formed from, sum p (|dP| + |delta|)."""
    rng = np.random.default_rng(23)
    att, dO = _case(rng, kind, 1, 2, 1, nq, nk, 48, 48, edges=edges, two_sided=two_sided, start=[start])
    Q, K, V, T, D = (_host(x)[0] if x.dim() == 4 else _host(x) for x in (att.Q, att.K, att.V, att.table, dO))
    want, size = np.zeros_like(T), np.zeros_like(T)
    b = A.bucket(np.arange(nk)[None, :] - np.arange(nq)[:, None] - start, edges, two_sided)
    for h in range(2):
        s = Q[:, h] @ K[:, 0].T * 48 ** -0.5 + T[h][b]
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        dP = D[:, h] @ V[:, 0].T
        delta = (p * dP).sum(1, keepdims=True)
        for n in range(T.shape[1]):
            want[h, n] = (p * (dP - delta))[b == n].sum()
            size[h, n] = (p * (np.abs(dP) + np.abs(delta)))[b == n].sum()
    O, lse = ctx.bbmm_attend(att)
    got = _host(ctx.bbmm_attend_grad(att, O, lse, dO)[3])
    off, lim = np.abs(got - want), A.UNIT[kind] * np.abs(want) + A.TINY[kind] + 64 * A.U32 * size
    assert (off <= lim).all(), (off / np.maximum(lim, 1e-300)).max()
