"""CPU checks of what the binding makes of arguments of other kinds than it takes, before any library call."""
import numpy as np
import pytest

from paper_1809_11165_amd import binding

torch = pytest.importorskip("torch")
CPU = torch.device("cpu")


def _rot(**kw):
    kw = {**dict(Q=torch.zeros(2, 5, 4, 8), K=torch.zeros(2, 5, 2, 8), pos=torch.zeros(2, 5, dtype=torch.int64), freq=torch.ones(3, dtype=torch.float64)), **kw}
    return binding.Rotation(**kw)


@pytest.mark.parametrize("axis", [3, 3.0, "012", np.array([0, 1, 0], np.float32), torch.zeros(3), [0, 1, 256], np.array([0]), torch.tensor(3)])
def test_axes_that_are_no_whole_numbers_are_refused(axis):
    with pytest.raises(ValueError, match="axis"):
        _rot(axis=axis).to_c(CPU)


@pytest.mark.parametrize("axis", [[0, 1, 0], (0, 1, 0), bytes([0, 1, 0]), np.array([0, 1, 0]), torch.tensor([0, 1, 0])])
def test_axes_as_any_sequence_of_whole_numbers(axis):
    r = _rot(axis=axis, pos=torch.zeros(2, 2, 5, dtype=torch.int64)).to_c(CPU)
    assert list(r.keep) == [0, 1, 0] and r.n_axes == 2


def test_an_axis_is_not_read_as_the_bytes_of_a_wider_number():
    with pytest.raises(ValueError, match="1 entries, expected 8"):
        _rot(axis=np.array([1]), Q=torch.zeros(2, 5, 4, 16), K=None, freq=torch.ones(8, dtype=torch.float64)).to_c(CPU)


@pytest.mark.parametrize("change,match", [
    (dict(eps="x"), "eps"), (dict(eps=[1e-6]), "eps"), (dict(pos=[[0] * 5] * 2), "pos"), (dict(pos=3), "pos"), (dict(freq=[1.0, 0.5, 0.1]), "freq"),
    (dict(freq=1.0), "freq"), (dict(freq=np.ones(3)), "freq"), (dict(freq=torch.tensor(1.0, dtype=torch.float64)), "freq"),
])
def test_rotations_of_no_numbers_and_no_tensors(change, match):
    with pytest.raises((TypeError, ValueError), match=match):
        _rot(**change).to_c(CPU)


@pytest.mark.parametrize("change", [dict(scale="x"), dict(scale=[0.1]), dict(cap=None), dict(cap="3"), dict(window=None), dict(window="x"),
                                    dict(window=float("inf")), dict(window=float("nan"))])
def test_cached_attentions_of_no_numbers(change):
    cache = binding.Cache(torch.zeros(6, 4, 2, 8), torch.zeros(6, 4, 2, 8), torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(TypeError, match="numbers"):
        binding.CachedAttention(cache, torch.zeros(2, 1, 4, 8), torch.zeros(2, dtype=torch.int32), **change).to_c(CPU)
