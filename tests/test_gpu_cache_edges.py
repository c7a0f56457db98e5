"""GPU parity of the attention over a paged cache where numbers are out of the ordinary: weights whose lowest bits decide, caps
from far below the scores to fp32's largest numbers."""
import numpy as np
import pytest

from oracle import cache_oracle as A
from test_gpu_cache import DEV, TYPES, _attend_and_check, _filled, _host, _int, _new, _rand

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_1809_11165_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_all_bits_of_a_weight_count_where_values_cancel(ctx, held):
    """Values of which less than 2^-10 of the size is left over, so that the output's own rounding is far below what weights of 16 bits would miss.

    A weight is off by less than 8 u32 (2 |s| log2 e for the steps before the exponential, 2 for it, 1 for its parts), the sums of n terms and the
    division by less than n + 2: (n + 10) u32 sum p|v|, and the output's own rounding."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(20)
    B, n, H, page = 32, 8, 16, 16

    def kept(x):                                           # what the cache holds of single-feature rows
        x = torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()
        return x if held == "bf16" else A.quantise(x[..., None])[0][..., 0]

    k = kept(-rng.random((B, n, H)))
    v = kept(rng.uniform(0.5, 1.5, (B, n, H)) * np.where(np.arange(n) % 2, 1, -1)[None, :, None])
    p = np.exp(k)
    p /= p.sum(1, keepdims=True)
    v[:, 4:] = 0
    for j in range(4, n):                                  # each of these cancels what is left
        v[:, j] = kept(-(p * v).sum(1) / p[:, j])
    pages, table = B, torch.arange(B, dtype=torch.int32, device=DEV)[:, None].contiguous()
    c = _new(held, pages, page, H, 1, 1, table, 0)
    as_rows = lambda x: torch.from_numpy(x).to(DEV).bfloat16()[..., None]
    ctx.bbmm_cache_write(c, as_rows(k), as_rows(v))
    Q = torch.ones(B, 1, H, 1, dtype=torch.bfloat16, device=DEV)
    O, _ = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([n] * B), scale=1.0))
    o = (p * v).sum(1)
    lim = (n + 10) * A.U32 * (p * np.abs(v)).sum(1) + A.UNIT["bf16"] * np.abs(o)
    most = np.abs(o).max()
    assert most < 2.0 ** -10
    worst = (np.abs(_host(O)[:, 0, :, 0] - o) / lim).max()
    assert worst <= 1


@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("cap", [1e-3, 0.3, 1e3, 1e5, 1e7, 1e9, 1e30, 1e38])
def test_caps_of_any_size(ctx, kind, held, cap):
    """A cap far above the scores leaves them as they are, one far below makes them plus or minus itself."""
    rng = np.random.default_rng(21)
    for shape in ((4, 1), (8, 5)):
        k_len = [300, 90]
        c = _filled(rng, kind, kind if held == "own" else held, k_len, 16, 2, 64, 64)
        Q = _rand(rng, kind, 2, shape[1], shape[0], 64, spread=3.0)
        _attend_and_check(ctx, kind, c, Q, k_len, cap=cap)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [0.01, 1.0, 50.0, 1e4, 1e20, 1e38])
def test_a_capped_score_is_as_exact_as_it_is_small(ctx, kind, cap):
    """Sequences of one key: lse is the score itself, which has to keep its relative error whatever its size beside the cap.

    Off by less than 10 u32 for the tanh and its factors (see the oracle), 1 for the product of the features and 2 for the way from the base-2 exponent to e: 13 u32,
    and steps of fp32's smallest numbers."""
    from paper_1809_11165_amd import binding
    B, H = 2048, 16
    n = B * H
    size = np.concatenate([np.linspace(0.4, 0.6, n // 4), np.geomspace(1e-6, 30, n - n // 4)]) * min(cap, 1e3)
    k = torch.from_numpy((size * np.where(np.arange(n) % 2, 1, -1)).astype(np.float32)).to(TYPES[kind]).view(B, 1, H, 1)
    c = _new(kind, B, 16, H, 1, 1, torch.arange(B, dtype=torch.int32, device=DEV)[:, None].contiguous(), 0)
    ctx.bbmm_cache_write(c, k.to(DEV), torch.ones_like(k, device=DEV))
    Q = torch.ones(B, 1, H, 1, dtype=TYPES[kind], device=DEV)
    _, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([1] * B), scale=1.0, cap=cap))
    s = cap * np.tanh(_host(k)[:, 0, :, 0] / cap)
    worst = (np.abs(_host(lse)[:, :, 0] - s) / (13 * A.U32 * np.abs(s) + 2.0 ** -140)).max()
    assert worst <= 1
