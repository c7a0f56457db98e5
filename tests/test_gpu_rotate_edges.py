"""GPU checks of the weights' gradients of the rotation to the last bit: rows of plus and minus one, whose norm is one, and whole numbers as gradients, so
that every sum is exact and a row left out or taken twice shows."""
import numpy as np
import pytest

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


# B, rows, HQ, HK, d, lengths: one workgroup, parts, several rounds, uneven shares, pieces of 16 bytes and single elements
SUMS = {
    "one_token": (1, 1, 4, 4, 64, None),
    "one_workgroup": (1, 15, 4, 4, 96, None),
    "one_workgroup_and_parts": (1, 40, 8, 1, 128, None),
    "a_part_a_token": (1, 37, 30, 2, 64, None),
    "many_tokens": (2, 3001, 2, 1, 32, None),
    "more_than_a_round": (1, 20011, 1, 1, 16, None),
    "several_rounds": (3, 7001, 4, 2, 128, None),
    "odd_features": (2, 5003, 3, 2, 33, None),
    "many_heads": (1, 50, 300, 1, 64, None),
    "only_queries": (2, 4001, 5, 0, 80, None),
    "lengths": (5, 2000, 4, 2, 64, [2000, 0, 1, 777, 1999]),
}


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("name", list(SUMS))
def test_every_row_counts_once(ctx, name, kind):
    from paper_1809_11165_amd import binding
    B, rows, HQ, HK, d, row_len = SUMS[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    live = np.ones((B, rows), bool) if row_len is None else np.arange(rows)[None] < np.array(row_len)[:, None]

    def made(heads):
        if not heads:
            return (None,) * 4
        x, g = rng.choice([-1.0, 1.0], (B, rows, heads, d)), rng.choice([-3.0, -1.0, 1.0, 3.0], (B, rows, heads, d))
        want = (x * g * live[:, :, None, None]).sum((0, 1, 2))
        to = lambda a: torch.from_numpy(a).to(DEV).to(TYPES[kind])
        return to(x), to(g), to(rng.standard_normal(d)), torch.from_numpy(want).to(torch.float32).to(TYPES[kind])

    (Q, dQ, wq, want_q), (K, dK, wk, want_k) = made(HQ), made(HK)
    rot = binding.Rotation(Q, K, None, None, eps=0.0, q_weight=wq, k_weight=wk,
                           row_len=None if row_len is None else torch.tensor(row_len, dtype=torch.int32, device=DEV))
    *_, gq, gk = ctx.bbmm_rotate_grad(rot, dQ, dK)
    for got, want in ((gq, want_q), (gk, want_k)):
        assert (got is None) == (want is None)
        assert got is None or torch.equal(got.cpu(), want)
