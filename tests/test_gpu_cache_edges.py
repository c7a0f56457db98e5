"""GPU parity of the attention over a paged cache where numbers are out of the ordinary: weights whose lowest bits decide, caps
from far below the scores to fp32's largest numbers, infinite values that some rows
take, and values whose sums leave fp32."""
import numpy as np
import pytest

from oracle import cache_oracle as A
from test_gpu_cache import DEV, TYPES, _attend_and_check, _bytes, _check, _filled, _host, _int, _new, _oracle, _rand

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    from paper_1809_11165_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("rows", [1, 32, 40])
@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_all_bits_of_a_weight_count_where_values_cancel(ctx, held, rows):
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
    Q = torch.ones(B, 1, rows * H, 1, dtype=torch.bfloat16, device=DEV)
    O, _ = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([n] * B), scale=1.0))
    o = (p * v).sum(1)
    lim = (n + 10) * A.U32 * (p * np.abs(v)).sum(1) + A.UNIT["bf16"] * np.abs(o)
    most = np.abs(o).max()
    assert most < 2.0 ** -10
    worst = (np.abs(_host(O).reshape(B, H, rows) - o[:, :, None]) / lim[:, :, None]).max()
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


# k_len, heads, hk, nq, d, dv, page, pages of a table row, options of the call; then the keys (sequence, from its end) whose value is not finite
ODD = {
    "one_row": ([300, 90], 4, 2, 1, 64, 64, 16, None, {}, [(0, 1), (0, 20), (0, 299), (1, 40)]),
    "one_row_page_of_twenty": ([300, 90], 4, 2, 1, 128, 128, 20, None, {}, [(0, 1), (0, 150), (1, 90)]),
    "new_rows": ([300, 90], 4, 2, 5, 64, 64, 16, None, {}, [(0, 1), (0, 3), (0, 150), (1, 4), (1, 89)]),
    "rows_40": ([300, 90], 8, 1, 5, 128, 128, 16, None, {}, [(0, 2), (0, 100), (0, 300), (1, 4), (1, 60)]),
    "rows_40_page_of_twenty": ([300, 90], 8, 1, 5, 128, 128, 20, None, {}, [(0, 2), (0, 100), (1, 3)]),
    "window": ([700, 90], 4, 2, 5, 64, 64, 16, None, dict(window=100), [(0, 3), (0, 50), (0, 102), (0, 104), (0, 300), (1, 85)]),
    "all_keys": ([300, 90], 4, 2, 5, 64, 64, 16, None, dict(causal=False), [(0, 1), (1, 40)]),
    "parts": ([5000, 1300], 4, 1, 1, 64, 64, 16, None, {}, [(0, 1), (0, 2500), (0, 4990), (1, 700)]),
    "parts_rows_40": ([5000, 1300], 8, 1, 5, 128, 128, 16, None, {}, [(0, 3), (0, 2500), (1, 700)]),
    "dealt": ([17000, 64, 700], 4, 2, 1, 64, 64, 16, 1100, {}, [(0, 9000), (1, 1), (2, 650)]),
    "odd_features": ([150, 90], 3, 1, 2, 33, 7, 16, None, {}, [(0, 1), (0, 100), (1, 50)]),
}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(ODD))
@pytest.mark.parametrize("value", ["inf", "-inf", "nan", "both"])
def test_infinite_values_come_through_where_they_are_taken(ctx, name, kind, value):
    """One feature of some values is infinite (or NaN, or infinities of both signs in turn): it is so in the outputs of the rows that take the key, wherever that
    lies among the blocks, and nothing else changes."""
    from paper_1809_11165_amd import binding
    k_len, heads, hk, nq, d, dv, page, most, opt, places = ODD[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    c = _filled(rng, kind, kind, k_len, page, hk, d, dv, most)
    Q = _rand(rng, kind, len(k_len), nq, heads, d)
    val, err = _oracle(kind, c, Q, k_len, **opt)
    for at, (b, back) in enumerate(places):
        j, f = k_len[b] - back, at % min(dv, 3)
        x = float(value) if value != "both" else (-1.0) ** (at // min(dv, 3)) * float("inf")
        c.V[int(c.table[b, j // page]), j % page, at % hk, f] = x
        takes = A.taken(k_len[b], nq, k_len[b], opt.get("causal", True), opt.get("window", 0))[:, j]
        heads_of = np.arange(heads) // (heads // hk) == at % hk
        with np.errstate(invalid="ignore"):
            val["o"][b, :, :, f][np.outer(takes, heads_of)] += x
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int(k_len), **opt))
    _check(lse, val, err, "lse")
    got = _host(O)
    off = ~np.isfinite(val["o"])
    assert off.any() and np.array_equal(got[off], val["o"][off], equal_nan=True)
    assert np.all(np.abs(got[~off] - val["o"][~off]) <= err["o"][~off])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [90, 5000])
@pytest.mark.parametrize("first", [True, False])
def test_an_infinite_value_whose_weight_rounds_to_zero(ctx, kind, n, first):
    """A weight is positive however small, in whatever order the keys come and whether or not they lie in one part.  The other values are those of the key that
    outweighs all, times its weight and divided by it: 4 u32, and rounded; lse is off by 4 u32 of itself (the factor to base 2 and back, twice rounded)."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(22)
    c = _filled(rng, kind, kind, [n], 16, 1, 64, 64)
    Q = torch.zeros(1, 1, 4, 64, dtype=TYPES[kind], device=DEV)
    Q[..., 0] = 16.0
    at = torch.arange(n, device=DEV)
    page, row = c.table[0].long()[at // 16], at % 16
    c.K[page, row, 0, 0] = 0.0
    far, top = (3, n - 3) if first else (n - 3, 3)
    c.K[page[top], row[top], 0, 0] = 100.0                   # 1600 above all others
    c.V[page[far], row[far], 0, 5] = float("inf")
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([n]), scale=1.0))
    want, got = _host(c.V[page[top], row[top], 0]), _host(O)[0, 0]
    assert np.all(got[:, 5] == np.inf)
    got[:, 5] = want[5]
    assert np.all(np.abs(got - want) <= (4 * A.U32 + A.UNIT[kind]) * np.abs(want))
    assert np.all(np.abs(_host(lse) - 1600) <= 4 * A.U32 * 1600)


@pytest.mark.parametrize("nq", [1, 5])
@pytest.mark.parametrize("back", [1, 200])
def test_8_bit_values_beyond_fp16_are_infinite_there(ctx, nq, back):
    """As they are where they are read back in fp16; in the other types they are numbers."""
    from paper_1809_11165_amd import binding
    for kind in TYPES:
        rng = np.random.default_rng(23)
        k_len = [300, 90]
        c = _filled(rng, kind, "e4m3", k_len, 16, 2, 64, 64)
        Q = _rand(rng, kind, 2, nq, 4, 64)
        j = k_len[0] - back
        page, row = int(c.table[0, j // 16]), j % 16
        c.V.view(torch.uint8)[page, row, :, :32] = 0x38      # ones
        c.v_exp[page, :, row, 0] = 127 + 17
        val, err = _oracle(kind, c, Q, k_len)
        if kind == "f16":
            takes = A.taken(300, nq, 300)[:, j]
            val["o"][0, takes, :, :32] = np.inf
        O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int(k_len)))
        _check(O, val, err, "o")
        _check(lse, val, err, "lse")


@pytest.mark.parametrize("kind,held", [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("k_len,heads,hk,nq,most,opt", [([300, 90], 4, 2, 1, None, {}), ([300, 90], 8, 1, 5, None, dict(cap=2.0)), ([700, 90], 4, 2, 3, None, dict(window=50)),
                                                        ([5000, 1300], 4, 1, 1, None, {}), ([17000, 64, 700], 4, 2, 1, 1100, {})])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 20)])
def test_means_of_values_whose_sums_leave_fp32(ctx, kind, held, k_len, heads, hk, nq, most, opt, d, page):
    """Values of 2^127: a sum of two is too large, a mean of any number is not."""
    rng = np.random.default_rng(24)
    c = _filled(rng, kind, held, k_len, page, hk, d, d, most)
    if held == "e4m3":
        c.V.view(torch.uint8).bitwise_and_(0x7f)
        c.v_exp.fill_(127 + 119)
    else:
        c.V.copy_(c.V.abs().clamp(0.5, 1) * 2.0 ** 127)
    Q = _rand(rng, kind, len(k_len), nq, heads, d)
    val, _ = _oracle(kind, c, Q, k_len, **opt)
    assert np.abs(val["o"]).max() > 2.0 ** (126 if held != "e4m3" else 118)
    _attend_and_check(ctx, kind, c, Q, k_len, **opt)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("k_len,page", [([300, 90], 16), ([300, 90], 5), ([5000, 1300], 16)])
def test_what_follows_the_last_feature_may_hold_anything(ctx, kind, held, k_len, page):
    """Pages that the caller has filled, up to each row's next 16 bytes, and exponents of blocks that are not there."""
    rng = np.random.default_rng(26)
    held = kind if held == "own" else held
    c = _filled(rng, kind, held, k_len, page, 2, 33, 7)
    Q = _rand(rng, kind, 2, 2, 4, 33)
    want = _oracle(kind, c, Q, k_len)
    for x, width in ((c.K, 33), (c.V, 7)):
        size = x.element_size()
        _bytes(x).view(-1, (width * size + 15) // 16 * 16)[:, width * size:] = 0x7f if held == "e4m3" else 0xff
    if held == "e4m3":
        c.k_exp[..., 2:], c.v_exp[..., 1:] = 255, 255
    _attend_and_check(ctx, kind, c, Q, k_len, want=want)


@pytest.mark.parametrize("bits", [0x7f800001, 0x7fc00000, -0x7fffff, -0x400000])
@pytest.mark.parametrize("held", ["f32", "e4m3"])
def test_a_query_of_any_nan_gives_nan(ctx, held, bits):
    """Also of one whose upper half is that of an infinity, which keys of one sign would make a score of -infinity."""
    from paper_1809_11165_amd import binding
    c = _filled(np.random.default_rng(25), "f32", held, [90], 16, 1, 64, 64)
    at = torch.arange(90, device=DEV)
    page, row = c.table[0].long()[at // 16], at % 16
    first = c.K.view(torch.uint8 if held == "e4m3" else torch.float32)
    first[page, row, 0, 0] = 0x38 if held == "e4m3" else 1.0
    for sign in (1, -1):
        if sign < 0:
            first[page, row, 0, 0] = 0xb8 if held == "e4m3" else -1.0
        Q = torch.zeros(1, 1, 2, 64, device=DEV)
        Q.view(torch.int32)[0, 0, 0, 0] = bits
        O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([90])))
        assert torch.isnan(O[0, 0, 0]).all() and torch.isnan(lse[0, 0]).all()
        assert torch.isfinite(O[0, 0, 1]).all() and torch.isfinite(lse[0, 1]).all()


def test_a_refusal_names_the_limit_that_is_passed(ctx):
    import ctypes as C
    from paper_1809_11165_amd import binding
    c = _new("f16", 1, 16, 1, 64, 64, torch.zeros(1, 1, dtype=torch.int32, device=DEV))
    s, a = binding.CachedAttention(c, torch.zeros(1, 1, 1, 64, dtype=torch.float16, device=DEV), _int([1])).to_c(ctx.device)
    n = C.c_int64(0)

    def refused(batch, kv_heads, heads, nq):
        s.batch, s.kv_heads, a.heads, a.nq = batch, kv_heads, heads, nq
        rc = ctx.lib.bbmm_attend_cache_workspace(ctx.h, C.byref(s), C.byref(a), C.byref(n))
        return None if rc == 0 else ctx.lib.bbmm_last_error(ctx.h).decode()

    assert refused(4096, 2048, 2048, 1) is None
    assert "2^23" in refused(4097, 2048, 2048, 1)          # 2^23 rows and as many blocks, each of a shared head of its own
    assert "2^23" in refused(4096, 4096, 4096, 1)
    assert refused(128, 1, 16, 65536) is None
    assert "2^27" in refused(129, 1, 16, 65536)
