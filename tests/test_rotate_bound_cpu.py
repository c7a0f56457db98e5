"""What the oracle's bound on the weights' gradients lets pass: not a row, a token or a workgroup that a sum leaves out or takes twice."""
import numpy as np
import pytest

from oracle import cache_oracle as A


@pytest.mark.parametrize("tokens,heads,d,left_out", [(20011, 1, 16, 20), (6002, 2, 32, 6), (6002, 2, 32, 1), (111, 8, 64, 1)])
def test_a_lost_part_of_a_sum_is_beyond_the_bound(tokens, heads, d, left_out):
    rng = np.random.default_rng(1)
    x, dy, w = rng.standard_normal((1, tokens, heads, d)), rng.standard_normal((1, tokens, heads, d)), rng.standard_normal(d)
    angle = rng.integers(0, 50, (1, tokens, 1)) * 10000.0 ** -(np.arange(d // 2) / (d // 2))
    val, err = A.rotate("f32", x, angle, eps=1e-6, weight=w, dy=dy)
    for first in (0, tokens // 2, tokens - left_out):
        some = slice(first, first + left_out)
        part, _ = A.rotate("f32", x[:, some], angle[:, some], eps=1e-6, weight=w, dy=dy[:, some])
        assert (np.abs(part["dw"]) > err["dw"]).mean() > 0.8
