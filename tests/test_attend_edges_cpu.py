"""CPU checks of the attention calls' boundary: inputs that torch's graph of gradients is to follow."""
import pytest

from paper_1809_11165_amd import binding

torch = pytest.importorskip("torch")


def test_inputs_that_require_grad_are_refused():
    """Before anything is queued; inside torch.no_grad() and for inputs that need none the call goes through."""
    class OnCpu:
        torch, device, _raw_stream = torch, torch.device("cuda", 0), None
    x, leaf = torch.zeros(2), torch.zeros(2, requires_grad=True)
    with pytest.raises(ValueError, match="requires grad"):
        binding.Context._ordered(OnCpu, [x, leaf], lambda: pytest.fail("queued"))
    raw = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None
    torch._C._cuda_getCurrentRawStream = lambda index: None
    try:
        assert binding.Context._ordered(OnCpu, [x], lambda: 1) == 1
        with torch.no_grad():
            assert binding.Context._ordered(OnCpu, [x, leaf], lambda: 2) == 2
    finally:
        if raw is None:
            del torch._C._cuda_getCurrentRawStream
        else:
            torch._C._cuda_getCurrentRawStream = raw
