"""GPU parity of the paged cache, written and read back, and of the attention that reads it, through the C ABI: bytes and values of the pages
(none but the written rows change), 8-bit rows against the format, attention against the fp64 oracle within the rounding bounds of
oracle/cache_oracle.py, over types, head sharing, page sizes and orders, missing pages, lengths, windows, garbage in places that take no part, far
offsets, streams and graphs; a sequence decoded token by token; and what the calls refuse."""
import numpy as np
import pytest

from oracle import cache_oracle as A

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
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


def _int(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def _table(rng, lens, page, most=None, spare=2):
    """(pages, table): scattered pages for sequences of these lengths, -1 behind them."""
    per = [(max(n, 0) + page - 1) // page for n in lens]
    most = max(per + [1]) if most is None else most
    pages = sum(per) + spare
    places = rng.permutation(pages)
    t, at = np.full((len(lens), most), -1, np.int32), 0
    for b, n in enumerate(per):
        t[b, :n] = places[at:at + n]
        at += n
    return pages, torch.from_numpy(t).to(DEV)


def _bytes(x):
    """The whole memory of a page tensor, pads among it, as bytes."""
    return torch.empty(0, dtype=torch.uint8, device=DEV).set_(x.untyped_storage())


def _new(held, pages, page, hk, d, dv, table, fill=0x5a):
    from paper_1809_11165_amd import binding
    c = binding.Cache.empty(pages, page, hk, d, dv, E4M3 if held == "e4m3" else TYPES[held], table, DEV)
    for x in (c.K, c.V, c.k_exp, c.v_exp):
        if x is not None:
            _bytes(x).fill_(fill)
    return c


# ---- written and read back --------------------------------------------------------------------------
# batch, rows, hk, d, dv, page, start, n_new
MOVES = {
    "one_row": (1, 1, 8, 128, 128, 16, [77], None),
    "one_row_each": (5, 1, 8, 128, 128, 16, [0, 15, 16, 100, 31], None),
    "chunk": (3, 50, 4, 64, 64, 16, [0, 13, 30], None),
    "odd_sizes": (2, 37, 3, 33, 7, 20, [5, 0], None),
    "one_feature": (2, 9, 2, 1, 1, 1, [3, 0], None),
    "page_of_one": (2, 11, 2, 40, 40, 1, [3, 0], None),
    "large_page": (2, 300, 2, 80, 96, 1000, [0, 650], None),
    "parts": (4, 20, 2, 64, 32, 16, [0, 5, 10, 3], [20, 0, 7, 1]),
    "parts_out_of_range": (3, 20, 2, 64, 32, 16, [0, 5, 10], [-3, 100, 20]),
    "many": (2, 2500, 2, 32, 128, 64, [11, 0], None),
}


@pytest.mark.parametrize("held", list(TYPES) + ["e4m3"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(MOVES))
def test_rows_written_and_read_back(ctx, name, kind, held):
    if held not in (kind, "e4m3"):
        return
    b, rows, hk, d, dv, page, start, n_new = MOVES[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    count = [rows] * b if n_new is None else [min(max(n, 0), rows) for n in n_new]
    pages, table = _table(rng, [s + rows for s in start], page)
    c = _new(held, pages, page, hk, d, dv, table)
    K, V = _rand(rng, kind, b, rows, hk, d), _rand(rng, kind, b, rows, hk, dv)
    before = [None if x is None else _bytes(x).clone() for x in (c.K, c.V, c.k_exp, c.v_exp)]
    ctx.bbmm_cache_write(c, K, V, _int(start), _int(n_new))
    # the same rows by torch, beside the memory as it was
    want = [None if x is None else x.clone() for x in before]
    size = c.K.element_size()
    for x, src, mem, exps in ((c.K, K, want[0], want[2]), (c.V, V, want[1], want[3])):
        width = src.shape[3]
        pitch = (width * size + 15) // 16 * 16
        mem = mem.view(pages, hk, page, pitch)
        for i in range(b):
            at = np.arange(start[i], start[i] + count[i])
            pg, row = table[i].cpu().numpy()[at // page], at % page
            if not len(at):
                continue
            new = src[i, :count[i]].transpose(0, 1).contiguous()     # (hk, row, width)
            if held == "e4m3":
                values, e = A.quantise(_host(new), kind)
                q = torch.from_numpy(values * np.exp2(-np.repeat(e, 32, -1)[..., :width].astype(float))).to(E4M3).to(DEV).view(torch.uint8)
                e = torch.from_numpy((e + 127).astype(np.uint8)).to(DEV)
            else:
                q = new.view(torch.uint8)
            full = torch.zeros(hk, len(at), pitch, dtype=torch.uint8, device=DEV)
            full[..., :width * size] = q
            for r in range(len(at)):
                mem[int(pg[r]), :, int(row[r])] = full[:, r]
                if exps is not None:
                    exps.view(pages, hk, page, 4)[int(pg[r]), :, int(row[r]), :e.shape[-1]] = e[:, r]
    for x, w in zip((c.K, c.V, c.k_exp, c.v_exp), want):
        if x is not None:
            assert torch.equal(_bytes(x), w)
    # back: what was written, from row 0 and from the middle
    length = [s + n for s, n in zip(start, count)]
    for first in (start, [s + n // 2 for s, n in zip(start, count)]):
        k, v = ctx.bbmm_cache_read(c, rows + 3, _int(first), _int(length), dtype=TYPES[kind])
        for got, src in ((k, K), (v, V)):
            assert got.shape == (b, rows + 3) + src.shape[2:]
            for i in range(b):
                new = _host(src[i])[first[i] - start[i]:count[i]]
                exact = A.quantise(new, kind)[0] if held == "e4m3" else new
                g = _host(got[i])
                assert np.array_equal(g[:len(exact)], exact) and not g[len(exact):].any()


def test_every_value_of_the_16_bit_types_in_8_bits(ctx):
    """All patterns, each 31 times beside a block's largest value of every size: infinities and NaN come back as NaN, all else as the format has it."""
    for kind in ("bf16", "f16"):
        every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[kind])
        top = torch.tensor([0.0, 1.75, 1.7578125, 2.0 ** -14, 447.0, 3.0 ** 9], dtype=torch.float32).to(TYPES[kind])
        blocks = torch.empty(6, 2048, 4, 32, dtype=TYPES[kind])
        for i in range(6):
            blocks[i] = every.view(2048, 1, 32)
            blocks[i, :, 1:, 0] = top[i]
            blocks[i, :, 2:, 1:] = blocks[i, :, 2:, 1:].flip(1)
        src = blocks.view(1, 6 * 2048, 1, 128).to(DEV)
        rows = src.shape[1]
        c = _new("e4m3", rows // 1024, 1024, 1, 128, 128, torch.arange(rows // 1024, dtype=torch.int32, device=DEV)[None])
        ctx.bbmm_cache_write(c, src, src)
        want, e = A.quantise(_host(src)[0, :, 0], kind)
        assert torch.equal(c.k_exp[:, 0].reshape(rows, 4), torch.from_numpy((e + 127).astype(np.uint8)).to(DEV))
        for dtype in (torch.float32, torch.bfloat16) + (() if kind == "bf16" else (torch.float16,)):
            for got in ctx.bbmm_cache_read(c, rows, dtype=dtype):
                value = want if dtype is not torch.float16 else torch.from_numpy(want).half().double().numpy()
                assert np.array_equal(_host(got)[0, :, 0], value, equal_nan=True)
                assert np.array_equal(np.isfinite(_host(got)[0, :, 0]), np.isfinite(_host(src)[0, :, 0]))


def test_every_8_bit_value_at_every_exponent(ctx):
    """Values of all codes times all powers that a cache holds: exact in fp32 and bf16; fp16 is the rounded one, infinite beyond its range."""
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    exps = torch.arange(10, 248, dtype=torch.int32).to(torch.uint8)            # 2^-117 .. 2^120
    rows = 2 * len(exps)
    c = _new("e4m3", 1, rows, 1, 128, 128, torch.zeros(1, 1, dtype=torch.int32, device=DEV))
    for x, e in ((c.K, c.k_exp), (c.V, c.v_exp)):
        x.view(torch.uint8)[0, :, 0] = codes.view(2, 128).repeat(len(exps), 1).to(DEV)
        e[0, 0] = exps.repeat_interleave(2)[:, None].expand(rows, 4).to(DEV)
    want = codes.view(E4M3).double().view(2, 128).repeat(len(exps), 1) * torch.exp2(exps.double() - 127).repeat_interleave(2)[:, None]
    for dtype in (torch.float32, torch.bfloat16):
        for got in ctx.bbmm_cache_read(c, rows, dtype=dtype):
            # (256 2^120 and more, which no write leaves, are beyond fp32 and infinite; everything else is the value itself)
            assert np.array_equal(_host(got)[0, :, 0], want.float().double().numpy(), equal_nan=True)
    for got in ctx.bbmm_cache_read(c, rows, dtype=torch.float16):
        assert np.array_equal(_host(got)[0, :, 0], want.float().half().double().numpy(), equal_nan=True)


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_missing_pages_and_rows_outside_the_table(ctx, held):
    rng = np.random.default_rng(1)
    b, hk, d, page = 4, 2, 64, 16
    table = torch.tensor([[0, -1, 2], [3, 9, 4], [2 ** 31 - 1, 5, -2 ** 31], [6, 7, 8]], dtype=torch.int32, device=DEV)     # pages 0 .. 8
    c = _new(held, 9, page, hk, d, d, table)
    K = _rand(rng, "bf16", b, 60, hk, d)
    start = [0, 0, -5, 40]
    ctx.bbmm_cache_write(c, K, K, _int(start))
    k, v = ctx.bbmm_cache_read(c, 70, _int([-3, 0, 0, 0]))
    assert torch.equal(k, v)
    exact = A.quantise(_host(K))[0] if held == "e4m3" else _host(K)
    got = _host(k)
    for i in range(b):
        for r in range(70):
            j = r + (-3 if i == 0 else 0)
            there = 0 <= j < 48 and 0 <= int(table[i, j // page]) < 9
            if not there:
                assert not got[i, r].any(), (i, r)
            elif start[i] <= j < start[i] + 60:
                assert np.array_equal(got[i, r], exact[i, j - start[i]]), (i, r)
    # nothing but rows 40 .. 47 of the last sequence in its page 8
    mem = _bytes(c.K).view(9, hk, page, -1)
    assert torch.all(mem[6:8] == 0x5a) and torch.all(mem[8, :, :8] == 0x5a) and not torch.all(mem[8, :, 8:] == 0x5a)
    # an empty table, no pages, no rows
    none = type(c)(c.K, c.V, table[:, :0].contiguous(), c.k_exp, c.v_exp)
    ctx.bbmm_cache_write(none, K, K)
    assert not ctx.bbmm_cache_read(none, 5)[0].any()
    gone = _new(held, 0, page, hk, d, d, table)
    ctx.bbmm_cache_write(gone, K, K)
    assert not ctx.bbmm_cache_read(gone, 5)[0].any()
    ctx.bbmm_cache_write(c, K[:, :0], K[:, :0])
    assert ctx.bbmm_cache_read(c, 0)[0].shape == (b, 0, hk, d)


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_first_pages_of_a_larger_allocation_and_strided_sources(ctx, kind):
    """Pages as (page, row, head, feature), keys and values side by side in one allocation of several layers."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(2)
    d, hk, page, b, rows = 48, 3, 8, 2, 21
    pages, table = _table(rng, [rows, rows], page)
    layers = torch.full((2, pages, page, hk, 2 * d), -9.0, dtype=TYPES[kind], device=DEV)
    c = binding.Cache(layers[1, ..., :d], layers[1, ..., d:], table)
    kv = _rand(rng, kind, b, rows, hk, 2 * d + 1)
    K, V = kv[..., :d], kv[..., d:2 * d]
    ctx.bbmm_cache_write(c, K, V)
    assert torch.all(layers[0] == -9)
    k, v = ctx.bbmm_cache_read(c, rows)
    assert torch.equal(k, K) and torch.equal(v, V)
    Q = _rand(rng, kind, b, 1, 2 * hk, d)
    _attend_and_check(ctx, kind, c, Q, [rows, rows - 4])


# ---- attention --------------------------------------------------------------------------------------
def _rows_of(c, total):
    """Keys and values of every sequence as fp64, and which rows' pages are there."""
    page = c.K.shape[1]
    table = c.table.cpu().numpy()
    at = np.arange(total)
    pg = table[:, at // page]
    there = (pg >= 0) & (pg < c.K.shape[0])
    pg = np.where(there, pg, 0)
    out = []
    for x, e in ((c.K, c.k_exp), (c.V, c.v_exp)):
        if e is not None:
            x = x.contiguous().view(torch.uint8).cpu().view(E4M3)
        v = _host(x)
        if e is not None:
            v = v * np.exp2(np.repeat(e.cpu().numpy().astype(float) - 127, 32, -1)[..., :v.shape[-1]].transpose(0, 2, 1, 3))
        out.append(np.where(there[:, :, None, None], v[pg, at % page], 0.0))
    return out[0], out[1], there


def _check(got, val, err, name):
    g = _host(got)
    assert g.shape == val[name].shape, name
    finite = np.isfinite(val[name])
    assert np.array_equal(g[~finite], val[name][~finite]), name
    assert np.all(np.isfinite(g[finite])), name
    off, lim = np.abs(g[finite] - val[name][finite]), err[name][finite]
    bad = off > lim
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its bound" % (name, bad.sum(), bad.size, (off[bad] / np.maximum(lim[bad], 1e-300)).max())


def _oracle(kind, c, Q, k_len, q_len=None, **kw):
    total = max([1] + [min(n, c.table.shape[1] * c.K.shape[1]) for n in k_len])
    K, V, there = _rows_of(c, total)
    return A.attend(kind, _host(Q), K, V, kw.pop("scale", Q.shape[3] ** -0.5), k_len, q_len, there=there, **kw)


def _attend_and_check(ctx, kind, c, Q, k_len, q_len=None, want=None, **kw):
    from paper_1809_11165_amd import binding
    val, err = want or _oracle(kind, c, Q, k_len, q_len, **kw)
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int(k_len), _int(q_len), **kw))
    _check(O, val, err, "o")
    _check(lse, val, err, "lse")
    return O, lse


def _filled(rng, kind, held, k_len, page, hk, d, dv, most=None, fill=0xff):
    """A cache of random rows; whatever is no row of a sequence (or a pad) keeps the bytes `fill` (NaN in all types)."""
    pages, table = _table(rng, k_len, page, most)
    c = _new(held, pages, page, hk, d, dv, table, fill)
    n = max([1] + list(k_len))
    K, V = _rand(rng, kind, len(k_len), n, hk, d), _rand(rng, kind, len(k_len), n, hk, dv)
    from paper_1809_11165_amd import binding
    writer = binding.Context(0)
    writer.bbmm_cache_write(c, K, V, None, _int(k_len))
    torch.cuda.synchronize()
    writer.close()
    return c


# k_len, heads, hk, nq, d, dv, page, options of the call
ATTEND = {
    "one_key": ([1], 1, 1, 1, 64, 64, 16, {}),
    "one_short": ([77], 4, 4, 1, 64, 64, 16, {}),
    "lengths": ([1, 31, 32, 33, 500, 0, 128], 8, 2, 1, 64, 64, 16, {}),
    "shared_long": ([3000, 1301], 8, 2, 1, 128, 128, 64, {}),
    "page_of_one": ([70, 129], 4, 2, 1, 64, 64, 1, {}),
    "page_of_twenty": ([333, 50], 6, 2, 3, 128, 128, 20, {}),
    "page_of_48": ([333, 50], 4, 4, 2, 40, 40, 48, {}),
    "large_page": ([900, 1700], 4, 2, 1, 96, 96, 2000, {}),
    "odd_features": ([150, 90], 3, 1, 2, 33, 7, 16, {}),
    "odd_features_page_of_five": ([150, 90], 3, 1, 2, 33, 7, 5, {}),
    "features_17_128": ([64, 65], 2, 2, 1, 17, 128, 32, {}),
    "one_feature": ([40], 2, 1, 1, 1, 1, 16, {}),
    "sixteen_rows": ([200], 16, 1, 1, 64, 64, 16, {}),
    "seventeen_rows": ([200], 17, 1, 1, 64, 64, 16, {}),
    "many_rows": ([200, 64], 40, 2, 5, 32, 32, 16, {}),
    "new_rows": ([100, 64, 9], 4, 2, 8, 64, 64, 16, {}),
    "more_new_rows_than_keys": ([3, 10], 4, 2, 8, 64, 64, 16, {}),
    "padded_new_rows": ([100, 64, 9], 4, 2, 8, 64, 64, 16, dict(q_len=[3, 8, 0])),
    "lengths_out_of_range": ([50, 40], 4, 2, 4, 64, 64, 16, dict(q_len=[-3, 100])),
    "all_keys": ([100, 64], 4, 2, 8, 64, 64, 16, dict(causal=False)),
    "window": ([2500, 100, 7], 4, 2, 1, 64, 64, 16, dict(window=50)),
    "window_of_one": ([90, 100], 4, 2, 3, 64, 64, 16, dict(window=1)),
    "window_new_rows": ([700, 333], 4, 1, 7, 128, 128, 32, dict(window=33)),
    "window_all_keys": ([300, 90], 4, 2, 5, 64, 64, 16, dict(window=40, causal=False)),
    "window_wider_than_all": ([300, 90], 4, 2, 5, 64, 64, 16, dict(window=2 ** 40)),
    "cap": ([300, 90], 4, 2, 2, 64, 64, 16, dict(cap=1.5)),
    "cap_window": ([700, 90], 4, 2, 2, 128, 128, 16, dict(cap=30.0, window=100)),
    "scale": ([300, 90], 4, 2, 2, 64, 64, 16, dict(scale=1.7)),
    "prompt": ([260, 200], 4, 1, 200, 64, 64, 64, dict(q_len=[200, 150])),
    "rows_33_page_of_twenty": ([333, 50], 11, 1, 3, 128, 128, 20, {}),
    "rows_40_cap": ([700, 130], 8, 1, 5, 100, 120, 32, dict(cap=3.0)),
    "rows_320_window": ([900, 41, 300], 32, 2, 20, 128, 128, 16, dict(window=70, q_len=[20, 20, 13])),
}


@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(ATTEND))
def test_attention_over_pages_matches_the_oracle(ctx, name, kind, held):
    k_len, heads, hk, nq, d, dv, page, opt = ATTEND[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    c = _filled(rng, kind, kind if held == "own" else held, k_len, page, hk, d, dv)
    _attend_and_check(ctx, kind, c, _rand(rng, kind, len(k_len), nq, heads, d), k_len, **opt)


# Tables wide enough that the keys of several sequences are cut by what their lengths are, not by the table's width.
def _short(b, most, **long):
    """b lengths up to `most`, some of them zero, but for {"at<number>": length}."""
    rng = np.random.default_rng(b)
    n = [int(x) for x in rng.integers(0, most + 1, b) * (rng.random(b) < 0.9)]
    for k, x in long.items():
        n[int(k[2:])] = x
    return n


# k_len, heads, hk, nq, d, dv, page, pages of a table row, options of the call
DEALT = {
    "a_long_and_a_short": ([17000, 3], 4, 2, 1, 64, 64, 16, 1100, {}),
    "a_short_and_a_long": ([3, 17000], 4, 2, 1, 64, 64, 16, 1100, {}),
    "all_short": ([1, 0, 40, 500, 64], 4, 2, 1, 64, 64, 16, 1100, {}),
    "all_empty": ([0, 0, 0], 4, 2, 1, 64, 64, 16, 1100, {}),
    "one_has_all": ([0, 0, 20000, 0], 4, 1, 1, 128, 128, 64, 320, {}),
    "equal": ([4100] * 4, 4, 1, 1, 64, 64, 16, 1100, {}),
    "lengths_out_of_range": ([-5, 2 ** 31 - 1, 700], 2, 1, 1, 32, 32, 4096, 5, dict(oracle=[0, 20480, 700])),
    "sixty_three": (_short(63, 300, at0=4000), 2, 1, 1, 32, 32, 16, 1100, {}),
    "sixty_four": (_short(64, 300, at63=4000), 2, 1, 1, 32, 32, 16, 1100, {}),
    "sixty_five": (_short(65, 300, at64=4000, at1=0), 2, 1, 1, 32, 32, 16, 1100, {}),
    "hundred_and_thirty": (_short(130, 300, at0=0, at129=3000, at64=2000), 2, 1, 1, 32, 32, 16, 1100, {}),
    "two_hundred_and_fifty_six": (_short(256, 200, at255=2500, at128=2000), 2, 1, 1, 32, 32, 16, 1100, {}),
    "two_hundred_and_fifty_seven": (_short(257, 200, at256=2500), 2, 1, 1, 32, 32, 16, 1100, {}),
    "as_many_as_fill_the_device": (_short(128, 200, at5=2500), 6, 6, 1, 16, 16, 16, 300, {}),
    "many_as_fill_the_device": (_short(256, 150, at0=2000, at255=0), 6, 3, 1, 16, 16, 16, 300, {}),
    "new_rows": ([17000, 64, 9], 4, 2, 8, 64, 64, 16, 1100, {}),
    "padded_new_rows": ([17000, 64, 9, 50, 0], 8, 1, 9, 64, 64, 16, 1100, dict(q_len=[9, 3, 0, -2, 9])),
    "new_rows_all_keys": ([3000, 64, 9], 8, 1, 9, 128, 128, 16, 1100, dict(causal=False)),
    "window": ([18000, 17100, 5, 0], 4, 1, 2, 64, 64, 32, 600, dict(window=17000)),
    "page_of_twenty": ([5000, 333, 50], 6, 2, 3, 128, 128, 20, 900, {}),
    "odd_features_page_of_five": ([2000, 90], 3, 1, 2, 33, 7, 5, 3400, {}),
    "cap": ([3000, 90], 4, 2, 2, 64, 64, 16, 1100, dict(cap=1.5)),
    "missing_pages": ([3000, 90, 32, 700], 4, 2, 2, 64, 64, 32, 600, dict(holes=True)),
    "missing_pages_of_five": ([3000, 90, 5, 700], 4, 2, 2, 64, 64, 5, 3400, dict(holes=True)),
}


@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(DEALT))
def test_keys_cut_by_all_lengths_match_the_oracle(ctx, name, kind, held):
    from paper_1809_11165_amd import binding
    k_len, heads, hk, nq, d, dv, page, most, opt = DEALT[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    opt = dict(opt)
    there, holes = opt.pop("oracle", k_len), opt.pop("holes", False)
    c = _filled(rng, kind, kind if held == "own" else held, there, page, hk, d, dv, most)
    if holes:
        c.table[:, ::3] = -1                                 # and the first page of each: one sequence is left without keys
    Q = _rand(rng, kind, len(k_len), nq, heads, d)
    want = _oracle(kind, c, Q, there, **opt)
    first = _attend_and_check(ctx, kind, c, Q, k_len, want=want, **opt)
    again = _attend_and_check(ctx, kind, c, Q, k_len, want=want, **opt)
    assert all(torch.equal(x, y) for x, y in zip(first, again))


@pytest.mark.parametrize("held", ["own", "e4m3"])
def test_a_recorded_call_cuts_the_keys_by_the_lengths_of_each_replay(held):
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(14)
    full = [16500, 300, 4000, 1]
    c = _filled(rng, "bf16", "bf16" if held == "own" else held, full, 16, 2, 64, 64)
    Q, n = _rand(rng, "bf16", 4, 2, 4, 64), _int([2, 2, 2, 1])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, n))
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, n))
        for now in ([16500, 300, 4000, 1], [0, 0, 0, 0], [5, 300, 0, 1], [16500, 0, 0, 0], [900, 20, 4000, 0]):
            n.copy_(_int(now))
            g.replay()
            stream.synchronize()
            eager = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, n))
            stream.synchronize()
            assert torch.equal(O, eager[0]) and torch.equal(lse, eager[1]), now
            val, err = _oracle("bf16", c, Q, now)
            _check(O, val, err, "o")
            _check(lse, val, err, "lse")
        del g
    ctx.close()


@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("page", [16, 32, 5])
def test_missing_pages_take_no_part(ctx, kind, held, page):
    rng = np.random.default_rng(3)
    k_len = [330, 100, 64]
    c = _filled(rng, kind, kind if held == "own" else held, k_len, page, 2, 64, 64)
    c.table[0, 1], c.table[0, 2], c.table[0, 5] = -1, c.K.shape[0], 2 ** 31 - 1
    c.table[1, :] = -2 ** 31                                # a sequence that nothing is left of
    Q = _rand(rng, kind, 3, 2, 4, 64)
    O, lse = _attend_and_check(ctx, kind, c, Q, k_len)
    assert torch.all(O[1] == 0) and torch.all(lse[1] == -float("inf"))
    _attend_and_check(ctx, kind, c, Q, k_len, window=page + 40)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("held", ["own", "e4m3"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_garbage_in_places_that_some_rows_do_not_take(ctx, kind, held, value):
    """Keys and values of a sequence's last rows, which its earlier new rows do not take, and of rows before the window."""
    rng = np.random.default_rng(4)
    k_len, nq, w = [100, 45], 5, 30
    c = _filled(rng, kind, kind if held == "own" else held, k_len, 16, 2, 64, 64)
    Q = _rand(rng, kind, 2, nq, 4, 64)
    want = _oracle(kind, c, Q, k_len, window=w)

    def put(x, b, j, what):
        page, row = int(c.table[b, j // 16]), j % 16
        if held == "e4m3":
            x.view(torch.uint8)[page, row] = 0x7f
        else:
            x[page, row] = what

    for b, n in enumerate(k_len):
        put(c.K, b, n - 2, value)
        put(c.V, b, n - 1, value)
        for x in (c.K, c.V):
            put(x, b, n - nq - w, value)
    from paper_1809_11165_amd import binding
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int(k_len), window=w))
    # rows up to the third (of five) take neither the key n - 2 nor the value n - 1
    _check(O[:, :3], {"o": want[0]["o"][:, :3]}, {"o": want[1]["o"][:, :3]}, "o")
    _check(lse[:, :, :3], {"lse": want[0]["lse"][:, :, :3]}, {"lse": want[1]["lse"][:, :, :3]}, "lse")
    last = O[:, 4].float()
    assert not torch.isfinite(last).any()                    # and the last one takes both
    # only the value: what a row takes of it comes through
    c2 = _filled(np.random.default_rng(4), kind, kind if held == "own" else held, k_len, 16, 2, 64, 64)
    c = c2
    for b, n in enumerate(k_len):
        put(c.V, b, n - 1, value)
    O, _ = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int(k_len), window=w))
    _check(O[:, :4], {"o": want[0]["o"][:, :4]}, {"o": want[1]["o"][:, :4]}, "o")
    if held == "own" and value == value:
        assert torch.all(O[:, 4].float() == value)
    else:
        assert torch.isnan(O[:, 4].float()).all()


@pytest.mark.parametrize("kind", list(TYPES))
def test_queries_that_take_no_part_may_hold_anything(ctx, kind):
    rng = np.random.default_rng(5)
    c = _filled(rng, kind, kind, [90, 70], 16, 2, 64, 64)
    Q = _rand(rng, kind, 2, 6, 4, 64)
    q_len = [2, 6]
    want = _oracle(kind, c, Q, [90, 70], q_len)
    Q[0, 2:] = float("nan")
    O, lse = _attend_and_check(ctx, kind, c, Q, [90, 70], q_len, want=want)
    assert torch.all(O[0, 2:] == 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("how", ["heads_first", "side_by_side", "off_by_one", "shared"])
def test_strides_and_alignments_of_queries(ctx, kind, how):
    rng = np.random.default_rng(6)
    c = _filled(rng, kind, kind, [90, 70], 16, 2, 64, 64)
    Q = _rand(rng, kind, 2, 3, 4, 64)
    if how == "heads_first":
        Q = Q.transpose(1, 2).contiguous().transpose(1, 2)
    elif how == "side_by_side":
        Q = torch.cat([Q, Q], 2)[:, :, 4:]
    elif how == "off_by_one":
        wide = torch.empty(Q.numel() + 1, dtype=Q.dtype, device=DEV)
        wide[1:] = Q.reshape(-1)
        Q = wide[1:].view(Q.shape)
    else:
        Q = Q[:1].expand(2, 3, 4, 64)
    _attend_and_check(ctx, kind, c, Q, [90, 70])


@pytest.mark.parametrize("kind", list(TYPES))
def test_scores_far_apart(ctx, kind):
    """Scores that rise along the keys, so that the reference of the softmax moves many times, and one that outweighs all."""
    rng = np.random.default_rng(7)
    c = _filled(rng, kind, kind, [400], 16, 1, 64, 64)
    Q = torch.zeros(1, 1, 2, 64, dtype=TYPES[kind], device=DEV)
    Q[0, 0, 0, 0], Q[0, 0, 1, 1] = 8.0, 8.0
    at = torch.arange(400, device=DEV)
    page, row = c.table[0].long()[at // 16], at % 16
    c.K[page, row, 0, 0] = (at * 0.25).to(TYPES[kind])
    c.K[page[123], row[123], 0, 1] = 400.0
    _attend_and_check(ctx, kind, c, Q, [400], scale=1.0)


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [64, 20])
def test_pages_beyond_32_bits_of_offset(ctx, held, page):
    """Pages at the end of an allocation of 5 GiB and more each for keys and values."""
    rng = np.random.default_rng(8)
    hk, d = 8, 128
    pages = 5 * 2 ** 30 // (hk * d * page * (2 if held == "bf16" else 1)) + 7
    table = torch.tensor([[pages - 1, 0, pages - 3], [pages // 2, pages - 2, 1]], dtype=torch.int32, device=DEV)
    from paper_1809_11165_amd import binding
    c = binding.Cache.empty(pages, page, hk, d, d, E4M3 if held == "e4m3" else torch.bfloat16, table, DEV)
    n = 3 * page
    K, V = _rand(rng, "bf16", 2, n, hk, d), _rand(rng, "bf16", 2, n, hk, d)
    ctx.bbmm_cache_write(c, K, V)
    k, v = ctx.bbmm_cache_read(c, n)
    exact = [A.quantise(_host(x))[0] if held == "e4m3" else _host(x) for x in (K, V)]
    assert np.array_equal(_host(k), exact[0]) and np.array_equal(_host(v), exact[1])
    Q = _rand(rng, "bf16", 2, 1, 16, d)
    val, err = A.attend("bf16", _host(Q), *exact, d ** -0.5, [n, n - 5])
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, _int([n, n - 5])))
    _check(O, val, err, "o")
    _check(lse, val, err, "lse")


@pytest.mark.parametrize("b,nq,most", [(0, 1, 3), (2, 0, 3), (2, 2, 0)])
def test_sizes_of_zero(ctx, b, nq, most):
    from paper_1809_11165_amd import binding
    c = _new("bf16", 4, 16, 2, 64, 64, torch.zeros(b, most, dtype=torch.int32, device=DEV))
    O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, torch.ones(b, nq, 4, 64, dtype=torch.bfloat16, device=DEV), _int([9] * b)))
    assert O.shape == (b, nq, 4, 64) and lse.shape == (b, 4, nq) and not O.any() and torch.all(lse == -float("inf"))


def test_a_sequence_decoded_token_by_token(ctx):
    """Norm, rotation, cache and attention as a server runs them: a prompt in one call, then single tokens; every row beside the
    attention over the whole sequence that is in memory as such."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(9)
    B, H, HK, d, page, prompt, total = 2, 8, 2, 64, 16, 37, 45
    freq = torch.from_numpy(10000.0 ** -(np.arange(32) / 32)).to(DEV)
    wq, wk = _rand(rng, "bf16", d), _rand(rng, "bf16", d)
    Q, K, V = _rand(rng, "bf16", B, total, H, d), _rand(rng, "bf16", B, total, HK, d), _rand(rng, "bf16", B, total, HK, d)
    pages, table = _table(rng, [total] * B, page)

    def turned(first, last):
        pos = torch.arange(first, last, device=DEV).expand(B, last - first).contiguous()
        return ctx.bbmm_rotate(binding.Rotation(Q[:, first:last], K[:, first:last], pos, freq, eps=1e-6, q_weight=wq, k_weight=wk))

    for held in ("bf16", "e4m3"):
        c = _new(held, pages, page, HK, d, d, table, 0xff)
        rows, at = [], 0
        for n in [prompt] + [1] * (total - prompt):
            q, k = turned(at, at + n)
            ctx.bbmm_cache_write(c, k, V[:, at:at + n], _int([at] * B))
            O, lse = ctx.bbmm_attend_cache(binding.CachedAttention(c, q, _int([at + n] * B)))
            rows.append((O, lse))
            at += n
        q, _ = turned(0, total)
        k, v = ctx.bbmm_cache_read(c, total, length=_int([total] * B))
        # everything ahead excluded by a table of -infinity
        edges = torch.zeros(H, 2, dtype=torch.bfloat16, device=DEV)
        edges[:, 1] = -float("inf")
        whole = binding.Attention(q, k, v, table=edges, edges=[])
        O, lse = ctx.bbmm_attend(whole)
        got = torch.cat([x for x, _ in rows], 1), torch.cat([x for _, x in rows], 2)
        for pair, once in ((got, False), ((O, lse), True)):
            val, err = A.attend("bf16", _host(q), _host(k), _host(v), d ** -0.5, [total] * B, once=once)
            _check(pair[0], val, err, "o")
            _check(pair[1], val, err, "lse")


def test_results_are_the_same_from_call_to_call_and_part_to_part(ctx):
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(10)
    c = _filled(rng, "bf16", "e4m3", [5000, 1234], 16, 2, 128, 128)
    att = binding.CachedAttention(c, _rand(rng, "bf16", 2, 1, 8, 128), _int([5000, 1234]))
    assert ctx.bbmm_attend_cache_workspace(att) > 0          # the keys are split
    want = ctx.bbmm_attend_cache(att)
    for _ in range(3):
        got = ctx.bbmm_attend_cache(att)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_another_stream_and_tensors_dropped_at_once(ctx):
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(11)
    c = _filled(rng, "bf16", "bf16", [700, 90], 16, 2, 64, 64)
    K, V, Q = _rand(rng, "bf16", 2, 4, 2, 64), _rand(rng, "bf16", 2, 4, 2, 64), _rand(rng, "bf16", 2, 4, 8, 64)
    start, k_len = _int([696, 86]), _int([700, 90])

    def step(context, K):
        context.bbmm_cache_write(c, K, V, start)
        return context.bbmm_attend_cache(binding.CachedAttention(c, Q, k_len)) + context.bbmm_cache_read(c, 700, length=k_len)

    want = step(ctx, K)
    torch.cuda.synchronize()
    other = binding.Context(0, stream=torch.cuda.Stream())
    try:
        for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
            ctx.bbmm_cache_write(c, torch.zeros_like(K), torch.zeros_like(V), start)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                late = torch.empty_like(K)
                torch.cuda._sleep(2_000_000)
                late.copy_(K)
                copies = [x.clone() for x in step(other, late)]
                del late
            stream.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(copies, want))
    finally:
        other.close()


def test_two_recorded_decode_steps_replayed_in_turn():
    """Two graphs of one context with caches and workspaces of their own, lengths that grow between the replays, eager work beside them."""
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(12)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        cases = []
        for held, n, hk, h in (("e4m3", [3000, 411], 2, 8), ("bf16", [90, 40], 4, 4)):
            c = _filled(rng, "bf16", held, [x + 8 for x in n], 16, hk, 64, 64)
            cases.append([c, _rand(rng, "bf16", 2, 1, h, 64), _rand(rng, "bf16", 2, 1, hk, 64), _rand(rng, "bf16", 2, 1, hk, 64), _int(n), _int([x + 1 for x in n])])

        def step(c, Q, K, V, start, k_len):
            ctx.bbmm_cache_write(c, K, V, start)
            return ctx.bbmm_attend_cache(binding.CachedAttention(c, Q, k_len))

        for x in cases:
            step(*x)
        stream.synchronize()
        graphs = []
        for x in cases:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = step(*x)
            graphs.append((g, out))
        for turn in range(4):
            for x in cases:
                for t in x[1:4]:
                    t.copy_(_rand(rng, "bf16", *t.shape))
                x[4].add_(1)
                x[5].add_(1)
            for g, _ in graphs:
                g.replay()
            eager = [step(*x) for x in cases]
            stream.synchronize()
            for (_, out), e in zip(graphs, eager):
                assert torch.equal(out[0], e[0]) and torch.equal(out[1], e[1]), turn
        del graphs
    ctx.close()


def test_two_contexts_at_work_at_once():
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(13)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [binding.Context(0, stream=s) for s in streams]
    cases = []
    for held, n in (("e4m3", [9000, 411]), ("bf16", [5000, 4000])):
        c = _filled(rng, "bf16", held, n, 16, 2, 128, 128)
        cases.append(binding.CachedAttention(c, _rand(rng, "bf16", 2, 1, 8, 128), _int(n)))
    torch.cuda.synchronize()
    want = []
    for k in (0, 1):
        with torch.cuda.stream(streams[k]):
            want.append(ctxs[k].bbmm_attend_cache(cases[k]))
        torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got.append((k, ctxs[k].bbmm_attend_cache(cases[k])))
    torch.cuda.synchronize()
    for k, out in got:
        assert torch.equal(out[0], want[k][0]) and torch.equal(out[1], want[k][1])
    for c in ctxs:
        c.close()


# ---- refusals ---------------------------------------------------------------------------------------
def test_refusals_of_the_library(ctx):
    import ctypes as C
    from paper_1809_11165_amd import binding
    rng = np.random.default_rng(14)
    c = _filled(rng, "f16", "f16", [40, 9], 16, 2, 64, 64)
    c8 = _filled(rng, "f16", "e4m3", [40, 9], 16, 2, 64, 64)
    Q, k_len = _rand(rng, "f16", 2, 1, 4, 64), _int([40, 9])
    K = _rand(rng, "f16", 2, 3, 2, 64)
    att = binding.CachedAttention(c, Q, k_len)
    O, lse = ctx.bbmm_attend_cache(att)
    stride = (C.c_int64 * 3)(*K.stride()[:3])
    why = lambda: ctx.lib.bbmm_last_error(ctx.h).decode()

    def changed(s, change):
        for name, x in change.items():
            setattr(s, name, x)
        return s

    def refused(needle, cache=c, **change):
        s = changed(cache.to_c(ctx.device), change)
        a = att.to_c(ctx.device)[1]
        assert ctx.lib.bbmm_attend_cache(ctx.h, C.byref(s), C.byref(a), O.data_ptr(), lse.data_ptr(), None, 0) == binding.EINVAL and needle in why(), change
        assert ctx.lib.bbmm_cache_write(ctx.h, C.byref(s), 1, 3, K.data_ptr(), stride, K.data_ptr(), stride, None, None) == binding.EINVAL and needle in why()
        assert ctx.lib.bbmm_cache_read(ctx.h, C.byref(s), 1, 3, None, None, K.data_ptr(), K.data_ptr()) == binding.EINVAL and needle in why()

    refused("type", type=4)
    refused("own type", type=2)
    refused("reserved", reserved=1)
    refused("kv_heads", batch=-1)
    refused("kv_heads", kv_heads=0)
    refused("pages", pages=-1)
    refused("pages", pages=1 << 31)
    refused("page_rows", page_rows=0)
    refused("page_rows", max_pages=1 << 27)
    refused("d and dv", d=129)
    refused("d and dv", dv=0)
    refused("required", K=None)
    refused("table", table=None)
    refused("required", cache=c8, K_exp=None)
    refused("16-byte", V=c.V.data_ptr() + 8)
    refused("16-byte", cache=c8, V_exp=c8.v_exp.data_ptr() + 4)
    refused("negative", k_stride=(C.c_int64 * 3)(0, -64, 0))
    refused("multiples", v_stride=(C.c_int64 * 3)(0, 60, 0))
    refused("2^21", v_stride=(C.c_int64 * 3)(0, 1 << 21, 0))

    def refused_att(needle, **change):
        s, a = att.to_c(ctx.device)
        changed(a, change)
        assert ctx.lib.bbmm_attend_cache(ctx.h, C.byref(s), C.byref(a), O.data_ptr(), lse.data_ptr(), None, 0) == binding.EINVAL and needle in why(), change

    refused_att("type", type=3)
    refused_att("own type", type=0)
    refused_att("kv_heads", heads=3)
    refused_att("heads", heads=0)
    refused_att("nq", nq=-1)
    refused_att("nq", nq=(1 << 20) + 1)
    refused_att("2^27", nq=1 << 20, heads=128)
    refused_att("window", window=-1)
    for s in (0.0, -1.0, float("inf"), float("nan"), 1e-60, 3e38):
        refused_att("scale", scale=s)
    for s in (-1.0, float("inf"), float("nan"), 1e-60, 3e38):
        refused_att("cap", cap=s)
    refused_att("required", Q=None)
    refused_att("required", k_len=None)
    refused_att("aligned", Q=Q.data_ptr() + 1)
    refused_att("aligned", k_len=k_len.data_ptr() + 2)
    refused_att("negative", q_stride=(C.c_int64 * 3)(-1, 0, 0))
    s, a = att.to_c(ctx.device)
    assert ctx.lib.bbmm_attend_cache(ctx.h, C.byref(s), C.byref(a), None, lse.data_ptr(), None, 0) == binding.EINVAL
    assert ctx.lib.bbmm_attend_cache(ctx.h, C.byref(s), None, O.data_ptr(), lse.data_ptr(), None, 0) == binding.EINVAL
    assert ctx.lib.bbmm_attend_cache(ctx.h, None, C.byref(a), O.data_ptr(), lse.data_ptr(), None, 0) == binding.EINVAL
    assert ctx.lib.bbmm_attend_cache(None, C.byref(s), C.byref(a), O.data_ptr(), lse.data_ptr(), None, 0) == binding.EINVAL
    for kind, k, st in ((3, K.data_ptr(), stride), (0, K.data_ptr(), stride), (1, None, stride), (1, K.data_ptr() + 1, stride), (1, K.data_ptr(), None)):
        assert ctx.lib.bbmm_cache_write(ctx.h, C.byref(s), kind, 3, k, st, K.data_ptr(), stride, None, None) == binding.EINVAL
    assert ctx.lib.bbmm_cache_write(ctx.h, C.byref(s), 1, 1 << 26, K.data_ptr(), stride, K.data_ptr(), stride, None, None) == binding.EINVAL and "2^27" in why()
    assert ctx.lib.bbmm_cache_write(ctx.h, C.byref(s), 1, 3, K.data_ptr(), stride, K.data_ptr(), stride, k_len.data_ptr() + 1, None) == binding.EINVAL
    assert ctx.lib.bbmm_cache_read(ctx.h, C.byref(s), 1, -1, None, None, K.data_ptr(), K.data_ptr()) == binding.EINVAL
    # a workspace: too small, missing, not aligned
    long = binding.CachedAttention(_filled(rng, "f16", "f16", [5000, 9], 16, 2, 64, 64), Q, _int([5000, 9]))
    need = ctx.bbmm_attend_cache_workspace(long)
    assert need > 0
    room = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
    s, a = long.to_c(ctx.device)
    for ptr, n in ((room.data_ptr(), need - 1), (None, need), (room.data_ptr() + 4, need)):
        assert ctx.lib.bbmm_attend_cache(ctx.h, C.byref(s), C.byref(a), O.data_ptr(), lse.data_ptr(), ptr, n) == binding.EINVAL and "workspace" in why()
    again = ctx.bbmm_attend_cache(att)
    assert torch.equal(again[0], O) and torch.equal(again[1], lse)
