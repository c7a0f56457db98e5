"""GPU parity of the bucketed bias as a matrix (equal to the table's entries, no rounding) and of its table's gradient, and a run of the
bias, the attention that adds it and both gradients together."""
import numpy as np
import pytest

from oracle import attend_oracle as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"
EDGES = [1, 2, 3, 4, 6, 9, 14, 21]
SIZES = [(1, 1, 1, 1), (2, 3, 1, 50), (2, 1, 37, 1), (1, 2, 63, 129), (3, 2, 70, 200), (1, 1, 300, 33), (2, 2, 5, 3001)]


@pytest.fixture(scope="module")
def ctx():
    from paper_1809_11165_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


def _host(x):
    return x.detach().to("cpu").to(torch.float64).numpy()


def _rand(rng, kind, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV).to(TYPES[kind])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("edges,two_sided", [(EDGES, True), (EDGES, False), ([], True), ([], False), ([1, 30, 1024], True), (list(range(1, 64)), True)])
@pytest.mark.parametrize("start", [0, 17, -40, 1 << 40])
def test_matrix_and_gradient(ctx, kind, edges, two_sided, start):
    rng = np.random.default_rng(1)
    for b, h, nq, nk in SIZES:
        table = _rand(rng, kind, h, (len(edges) + 1) * (2 if two_sided else 1))
        B = ctx.bbmm_bucket_bias(table, edges, nq, nk, two_sided=two_sided, start=start)
        assert np.array_equal(_host(B), A.bias_matrix(_host(table), edges, two_sided, start, nq, nk))
        dB = _rand(rng, kind, b, h, nq, nk)
        got = _host(ctx.bbmm_bucket_bias_grad(dB, edges, two_sided=two_sided, start=start))
        val, mag = A.table_grad(_host(dB), edges, two_sided, start)
        # sums of at most nq rows and nk columns one after the other in fp32, rounded to the type once
        assert np.all(np.abs(got - val) <= (nq + nk) * A.U32 * mag + A.UNIT[kind] * np.abs(val) + A.TINY[kind])


def test_special_entries_come_through(ctx):
    table = torch.tensor([[float("-inf"), float("nan"), float("inf"), -0.0]], device=DEV)
    B = _host(ctx.bbmm_bucket_bias(table, [2], 9, 9))
    want = A.bias_matrix(table.cpu().numpy(), [2], True, 0, 9, 9)
    assert np.array_equal(B, want, equal_nan=True) and np.array_equal(np.signbit(B), np.signbit(want))


@pytest.mark.parametrize("kind", list(TYPES))
def test_no_rows_or_columns(ctx, kind):
    for b, h, nq, nk in ((0, 2, 3, 4), (2, 2, 0, 4), (2, 2, 3, 0)):
        assert ctx.bbmm_bucket_bias(_rand(np.random.default_rng(2), kind, h, 18), EDGES, nq, nk).shape == (h, nq, nk)
        dT = ctx.bbmm_bucket_bias_grad(torch.empty(b, h, nq, nk, dtype=TYPES[kind], device=DEV), EDGES)
        assert dT.shape == (h, 18) and torch.all(dT == 0)


def test_every_call_gives_the_same_bits(ctx):
    dB = _rand(np.random.default_rng(3), "f32", 3, 4, 200, 700)
    first = ctx.bbmm_bucket_bias_grad(dB, EDGES)
    assert all(torch.equal(first, ctx.bbmm_bucket_bias_grad(dB, EDGES)) for _ in range(3))


def test_refusals(ctx):
    from paper_1809_11165_amd import binding
    table = _rand(np.random.default_rng(4), "f32", 2, 18)
    with pytest.raises(ValueError):
        ctx.bbmm_bucket_bias(table, EDGES, 4, 4, two_sided=False)         # buckets of the other kind
    with pytest.raises(TypeError):
        ctx.bbmm_bucket_bias(table.double(), EDGES, 4, 4)
    with pytest.raises(ValueError):
        ctx.bbmm_bucket_bias(table.cpu(), EDGES, 4, 4)
    with pytest.raises(ValueError):
        ctx.bbmm_bucket_bias_grad(torch.zeros(1, 2, 8, 8, device=DEV).transpose(2, 3)[:, :, :4], EDGES)
    for edges in ([2, 2, 3, 4, 5, 6, 7, 8], [0, 2, 3, 4, 5, 6, 7, 8], [1, 2, 3, 4, 5, 6, 7, 1025]):
        with pytest.raises(binding.BbmmError) as e:
            ctx.bbmm_bucket_bias(table, edges, 4, 4)
        assert e.value.code == binding.EINVAL
    with pytest.raises(binding.BbmmError):
        ctx.bbmm_bucket_bias(table, EDGES, 4, 4, start=(1 << 40) + 1)
    with pytest.raises(binding.BbmmError):
        ctx.bbmm_bucket_bias_workspace(1, 1, 1 << 25, 4, 8)


@pytest.mark.parametrize("kind", list(TYPES))
def test_the_matrix_is_the_bias_that_the_attention_adds(ctx, kind):
    """The operators together, as a model uses them: values read off by attention with the table equal those of a softmax over scores
    plus the matrix, and the table's gradient is that of the matrix summed by bucket (both within their rounding bounds)."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(5)
    b, h, nq, nk, d, start = 2, 3, 90, 140, 32, 25
    edges = binding.bucket_edges(16, 40)
    Q, K, V, dO = (_rand(rng, kind, b, n, h, d) for n in (nq, nk, nk, nq))
    table = _rand(rng, kind, h, 16)
    att = binding.Attention(Q, K, V, table=table, edges=edges, q_start=torch.full((b,), start, dtype=torch.int64, device=DEV))
    O, lse = ctx.bbmm_attend(att)
    dT = ctx.bbmm_attend_grad(att, O, lse, dO)[3]
    B = _host(ctx.bbmm_bucket_bias(table, edges, nq, nk, start=start))
    val, err = A.attend(kind, _host(Q), _host(K), _host(V), d ** -0.5, dO=_host(dO), table=_host(table), edges=edges, start=[start] * b)
    s = np.einsum("bihd,bjhd->bhij", _host(Q), _host(K)) * d ** -0.5 + B[None]
    p = np.exp(s - s.max(3, keepdims=True))
    p /= p.sum(3, keepdims=True)
    o = np.einsum("bhij,bjhd->bihd", p, _host(V))
    assert np.all(np.abs(_host(O) - o) <= err["o"])
    dp = np.einsum("bihd,bjhd->bhij", _host(dO), _host(V))
    ds = p * (dp - (p * dp).sum(3, keepdims=True))
    dS = torch.from_numpy(ds.astype(np.float32)).to(DEV)
    by_matrix = _host(ctx.bbmm_bucket_bias_grad(dS, edges, start=start))
    mag = A.table_grad(ds, edges, True, start)[1]
    assert np.all(np.abs(_host(dT) - by_matrix) <= err["dtable"] + ((nq + nk) * A.U32 + A.U32) * mag)


@pytest.mark.parametrize("start", [1 << 64, (1 << 64) + 5, -(1 << 70)])
def test_starts_beyond_64_bits_are_refused(ctx, start):
    from paper_1809_11165_amd import binding
    table = _rand(np.random.default_rng(5), "f32", 2, 18)
    with pytest.raises(binding.BbmmError):
        ctx.bbmm_bucket_bias(table, EDGES, 4, 4, start=start)
    with pytest.raises(binding.BbmmError):
        ctx.bbmm_bucket_bias_grad(torch.zeros(1, 2, 4, 4, device=DEV), EDGES, start=start)
