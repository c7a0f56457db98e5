"""GPU parity of the attention over a paged cache where numbers are out of the ordinary: weights whose lowest bits decide."""
import numpy as np
import pytest

from oracle import cache_oracle as A
from test_gpu_cache import DEV, TYPES, _bytes, _check, _filled, _host, _int, _new, _oracle, _rand

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
