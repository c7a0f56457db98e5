"""CPU checks of the rotation's and the cache's boundary: struct layouts, argument checks of the binding (before any library call), the
division that kernels get from the host, and the fp64 oracle against automatic differentiation, differences and torch's 8-bit type."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle import cache_oracle as A
from paper_1809_11165_amd import binding

torch = pytest.importorskip("torch")
CPU = torch.device("cpu")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I32, I64, F64 = torch.int32, torch.int64, torch.float64


@pytest.mark.parametrize("name,struct", [("bbmm_rotation", binding._Rotation), ("bbmm_cache", binding._Cache),
                                         ("bbmm_cached_attention", binding._CachedAttention)])
def test_struct_layouts_match_the_header(name, struct):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bbmm.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text).group(1)
    want = {"int32_t": 4, "int64_t": 8, "double": 8, "*": 8}
    names, sizes = [], []
    for decl in filter(None, (x.strip() for x in body.split(";"))):
        kind = "*" if "*" in decl else decl.split()[0]
        for nm in re.sub(r"^(const\s+)?\w+\s*\**\s*", "", decl).split(","):
            m = re.match(r"\s*\**(\w+)(?:\[(\d+)\])?", nm)
            names.append(m.group(1))
            sizes.append(want[kind] * int(m.group(2) or 1))
    assert names == [f[0] for f in struct._fields_]
    assert sizes == [getattr(struct, f[0]).size for f in struct._fields_]


def test_division_by_a_number_from_the_host(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    exe = tmp_path / "div_sweep"
    subprocess.run([gxx, "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_1809_11165_amd", "csrc"),
                    os.path.join(ROOT, "tests", "div_sweep.cpp"), "-o", str(exe)], check=True)
    proc = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, timeout=300)
    assert proc.returncode == 0 and proc.stdout.startswith("ok "), proc.stdout


# ---- the binding ------------------------------------------------------------------------------------
def _rot(b=2, rows=5, h=4, hk=2, d=8, half=3, **kw):
    kw = {**dict(Q=torch.zeros(b, rows, h, d), K=torch.zeros(b, rows, hk, d), pos=torch.zeros(b, rows, dtype=I64),
                 freq=torch.ones(half, dtype=F64)), **kw}
    return binding.Rotation(**kw)


def test_a_rotation_carries_sizes_strides_and_defaults():
    qkv = torch.zeros(2, 5, 8, 8)
    r = _rot(Q=qkv[:, :, :4], K=qkv[:, :, 4:6]).to_c(CPU)
    assert (r.batch, r.rows, r.q_heads, r.k_heads, r.d, r.rot, r.n_axes, r.norm, r.neighbours) == (2, 5, 4, 2, 8, 6, 1, 0, 0)
    assert list(r.q_stride) == [320, 64, 8] and r.K == qkv.data_ptr() + 4 * 32
    r = _rot(pos=torch.zeros(3, 2, 5, dtype=I64), axis=[2, 0, 1], eps=0.0, neighbours=True, K=None).to_c(CPU)
    assert (r.n_axes, r.norm, r.eps, r.neighbours, r.k_heads, r.K) == (3, 1, 0.0, 1, 0, None)
    r = _rot(Q=None, pos=None, freq=None).to_c(CPU)
    assert (r.rot, r.q_heads, r.k_heads) == (0, 0, 2)


@pytest.mark.parametrize("change,error", [
    (dict(K=torch.zeros(2, 5, 2, 9)), ValueError),
    (dict(K=torch.zeros(2, 6, 2, 8)), ValueError),
    (dict(K=torch.zeros(2, 5, 2, 8, dtype=torch.float16)), TypeError),
    (dict(Q=torch.zeros(5, 4, 8)), ValueError),
    (dict(K=torch.zeros(5, 2, 8)), ValueError),
    (dict(Q=torch.zeros(2, 5, 4, 8, dtype=F64)), TypeError),
    (dict(Q=None, K=None), ValueError),
    (dict(Q=torch.zeros(2, 5, 4, 16)[..., ::2]), ValueError),
    (dict(pos=torch.zeros(2, 5, dtype=I32)), TypeError),
    (dict(pos=torch.zeros(2, 4, dtype=I64)), ValueError),
    (dict(pos=torch.zeros(1, 5, 2, dtype=I64)), ValueError),
    (dict(freq=torch.ones(3)), TypeError),
    (dict(freq=torch.ones(3, 1, dtype=F64)), ValueError),
    (dict(axis=[0, 0]), ValueError),
    (dict(axis=[0, 0, -1]), ValueError),
    (dict(axis=[0, 0, 0.5]), ValueError),
    (dict(q_weight=torch.ones(7), eps=1e-6), ValueError),
    (dict(k_weight=torch.ones(8, dtype=torch.bfloat16), eps=1e-6), TypeError),
    (dict(row_len=torch.zeros(2, dtype=I64)), TypeError),
    (dict(row_len=torch.zeros(3, dtype=I32)), ValueError),
])
def test_the_binding_refuses_rotations(change, error):
    with pytest.raises(error):
        _rot(**change).to_c(CPU)


def _cache(pages=6, rows=4, hk=2, d=8, dv=8, b=2, most=3, **kw):
    kw = {**dict(K=torch.zeros(pages, rows, hk, d), V=torch.zeros(pages, rows, hk, dv), table=torch.zeros(b, most, dtype=I32)), **kw}
    return binding.Cache(**kw)


def test_a_cache_carries_sizes_and_strides():
    c = binding.Cache.empty(6, 4, 2, 36, 20, torch.float16, torch.zeros(2, 3, dtype=I32), CPU)
    s = c.to_c(CPU)
    assert (s.type, s.pages, s.page_rows, s.kv_heads, s.d, s.dv, s.batch, s.max_pages) == (binding.TYPE_F16, 6, 4, 2, 36, 20, 2, 3)
    assert list(s.k_stride) == [320, 40, 160] and list(s.v_stride) == [192, 24, 96]     # rows from 16 bytes to 16 bytes
    c = binding.Cache.empty(6, 4, 2, 36, dtype=torch.float8_e4m3fn, table=torch.zeros(2, 3, dtype=I32), device=CPU)
    s = c.to_c(CPU)
    assert s.type == binding.TYPE_E4M3 and list(s.v_stride) == [384, 48, 192] and s.K_exp and s.V_exp
    c, a = binding.CachedAttention(_cache(), torch.zeros(2, 3, 4, 8), torch.zeros(2, dtype=I32)).to_c(CPU)
    assert (a.type, a.causal, a.heads, a.nq, a.window, a.cap, a.scale) == (binding.TYPE_F32, 1, 4, 3, 0, 0.0, 8 ** -0.5)


@pytest.mark.parametrize("change,error", [
    (dict(V=torch.zeros(6, 4, 1, 8)), ValueError),
    (dict(V=torch.zeros(5, 4, 2, 8)), ValueError),
    (dict(V=torch.zeros(6, 4, 2, 8, dtype=torch.float16)), TypeError),
    (dict(K=torch.zeros(6, 4, 8)), ValueError),
    (dict(K=torch.zeros(6, 4, 2, 8, dtype=F64)), TypeError),
    (dict(table=torch.zeros(2, 3, dtype=I64)), TypeError),
    (dict(table=torch.zeros(6, dtype=I32)), ValueError),
    (dict(table=None), ValueError),
    (dict(table=torch.zeros(3, 2, dtype=I32).T), ValueError),
    (dict(k_exp=torch.zeros(6, 2, 4, 4, dtype=torch.uint8)), ValueError),
])
def test_the_binding_refuses_caches(change, error):
    with pytest.raises(error):
        _cache(**change).to_c(CPU)


@pytest.mark.parametrize("change,error", [
    (dict(k_exp=None), ValueError),
    (dict(v_exp=torch.zeros(6, 4, 2, 4, dtype=torch.uint8)), ValueError),
    (dict(v_exp=torch.zeros(6, 2, 4, 4, dtype=torch.int8)), TypeError),
])
def test_the_binding_refuses_8_bit_caches(change, error):
    c = binding.Cache.empty(6, 4, 2, 8, dtype=torch.float8_e4m3fn, table=torch.zeros(2, 3, dtype=I32), device=CPU)
    for name, x in change.items():
        setattr(c, name, x)
    with pytest.raises(error):
        c.to_c(CPU)


@pytest.mark.parametrize("change,error", [
    (dict(Q=torch.zeros(3, 1, 4, 8)), ValueError),
    (dict(Q=torch.zeros(2, 1, 4, 9)), ValueError),
    (dict(Q=torch.zeros(2, 4, 8)), ValueError),
    (dict(Q=torch.zeros(2, 1, 4, 8, dtype=torch.bfloat16)), TypeError),
    (dict(k_len=torch.zeros(2, dtype=I64)), TypeError),
    (dict(k_len=None), TypeError),
    (dict(q_len=torch.zeros(1, dtype=I32)), ValueError),
])
def test_the_binding_refuses_cached_attentions(change, error):
    kw = {**dict(cache=_cache(), Q=torch.zeros(2, 1, 4, 8), k_len=torch.zeros(2, dtype=I32)), **change}
    with pytest.raises(error):
        binding.CachedAttention(**kw).to_c(CPU)


# ---- the oracle -------------------------------------------------------------------------------------
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_the_oracles_rotation_against_automatic_differentiation(neighbours, norm):
    rng = np.random.default_rng(1)
    B, rows, H, d, rot = 2, 4, 3, 9, 6
    x, dy, w = rng.standard_normal((B, rows, H, d)), rng.standard_normal((B, rows, H, d)), rng.standard_normal(d)
    pos = rng.integers(-50, 50, (2, B, rows))
    freq, axis, length = np.array([1.0, 0.3, 0.01]), [0, 1, 0], [4, 2]
    ang = A.angles(pos, freq, axis)
    kw = dict(eps=1e-3, weight=w) if norm else {}
    val, err = A.rotate("f32", x, ang, neighbours, dy=dy, row_len=length, **kw)
    tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    total = 0.0
    for b in range(B):
        for i in range(rows):
            if i >= length[b]:
                assert np.all(val["y"][b, i] == 0) and np.all(val["dx"][b, i] == 0) and np.all(err["dx"][b, i] == 0)
                continue
            for h in range(H):
                z = tx[b, i, h]
                if norm:
                    z = z / torch.sqrt((z * z).mean() + 1e-3) * tw
                y = [z[c] for c in range(d)]
                for p in range(3):
                    t = float(pos[axis[p], b, i] * freq[p])
                    c0, c1 = (2 * p, 2 * p + 1) if neighbours else (p, p + 3)
                    y[c0], y[c1] = z[c0] * np.cos(t) - z[c1] * np.sin(t), z[c1] * np.cos(t) + z[c0] * np.sin(t)
                y = torch.stack(y)
                assert np.allclose(val["y"][b, i, h], y.detach().numpy(), atol=1e-13)
                total = total + (y * torch.tensor(dy[b, i, h])).sum()
    total.backward()
    assert np.allclose(val["dx"], tx.grad.numpy(), atol=1e-12)
    if norm:
        assert np.allclose(val["dw"], tw.grad.numpy(), atol=1e-12)


def test_the_oracles_rotation_against_differences():
    rng = np.random.default_rng(2)
    x, dy, w = rng.standard_normal((1, 3, 2, 8)), rng.standard_normal((1, 3, 2, 8)), rng.standard_normal(8)
    ang = rng.standard_normal((1, 3, 4))
    val, _ = A.rotate("f32", x, ang, eps=1e-2, weight=w, dy=dy)
    for _ in range(5):
        ex, ew, h = rng.standard_normal(x.shape), rng.standard_normal(8), 1e-5
        up = (A.rotate("f32", x + h * ex, ang, eps=1e-2, weight=w + h * ew)[0]["y"] * dy).sum()
        down = (A.rotate("f32", x - h * ex, ang, eps=1e-2, weight=w - h * ew)[0]["y"] * dy).sum()
        want = (val["dx"] * ex).sum() + (val["dw"] * ew).sum()
        assert abs((up - down) / (2 * h) - want) < 1e-7 * (1 + abs(want))     # h^2 and 2^-52 / h


def test_the_oracles_8_bit_values_are_the_types():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    fine = every[np.isfinite(every)]
    assert np.array_equal(A.e4m3(fine), fine) and np.abs(fine).max() == 448
    rng = np.random.default_rng(3)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.02, (np.sort(fine)[1:] + np.sort(fine)[:-1]) / 2]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(A.e4m3(x), want)
    held, e = A.quantise(np.concatenate([np.full(32, 1.75), np.full(32, 1.7578125), np.zeros(32), [np.inf, np.nan, 3.0]])[None])
    assert e.tolist() == [[-8, -7, 0, -7]]
    assert np.array_equal(held[0, :64], [1.75] * 32 + [1.75] * 32) and np.isnan(held[0, 96:98]).all() and held[0, 98] == 3.0
    held, e = A.quantise(np.array([[1e-45, 2.0 ** -126, 0, 0]]))
    assert e[0, 0] == -117 and held[0].tolist() == [0, 2.0 ** -126, 0, 0]


@pytest.mark.parametrize("cap,window,causal", [(0.0, 0, True), (0.7, 0, False), (0.0, 3, True), (2.0, 2, False)])
def test_the_oracles_attention_against_the_formula(cap, window, causal):
    rng = np.random.default_rng(4)
    Q, K, V = rng.standard_normal((2, 3, 4, 5)), rng.standard_normal((2, 9, 2, 5)), rng.standard_normal((2, 9, 2, 6))
    there = rng.random((2, 9)) < 0.8
    val, err = A.attend("f32", Q, K, V, 0.4, [9, 2], q_len=[2, 3], causal=causal, window=window, cap=cap, there=there)
    for b, (n, ni) in enumerate(((9, 2), (2, 3))):
        for i in range(3):
            keys = [j for j in range(n) if there[b, j] and (not causal or j <= n - ni + i) and (not window or j > n - ni + i - window)]
            for h in range(4):
                if i >= ni or not keys:
                    assert np.all(val["o"][b, i, h] == 0) and val["lse"][b, h, i] == -np.inf
                    continue
                s = torch.tensor([0.4 * float(Q[b, i, h] @ K[b, j, h // 2]) for j in keys], dtype=F64)
                if cap:
                    s = cap * torch.tanh(s / cap)
                assert np.isclose(val["lse"][b, h, i], float(torch.logsumexp(s, 0)), atol=1e-13)
                assert np.allclose(val["o"][b, i, h], (torch.softmax(s, 0)[:, None] * torch.tensor(V[b, keys, h // 2])).sum(0).numpy(), atol=1e-13)
    assert all(np.all(e >= 0) for e in err.values())
