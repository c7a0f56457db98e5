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
