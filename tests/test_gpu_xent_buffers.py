"""The linear head's own buffers: when they are made, and by which calls."""
import pytest
import torch

from paper_2606_19025_amd.train import LinearCrossEntropy


def small(N=20, d=64, V=300):
    g = torch.Generator(device="cuda").manual_seed(N)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    return r(N, d), r(V, d) / 8, torch.randint(0, V, (N,), generator=g, device="cuda").int()


@pytest.mark.gpu
@pytest.mark.parametrize("fails", ["empty", "zeros"])
def test_a_backward_without_memory_can_be_called_again(gpu_lib, monkeypatch, fails):
    """One of the buffers does not fit: nothing is kept of the call, and the next one runs."""
    args = small()
    L = LinearCrossEntropy(20, 64, 300)
    L.forward(*args)

    def full(*a, **kw):
        raise torch.OutOfMemoryError("no memory")

    with monkeypatch.context() as m:
        m.setattr(torch, fails, full)
        with pytest.raises(torch.OutOfMemoryError):
            L.backward(*args, accumulate_dw=1)
    assert L.dx is None and L.dw is None
    M = LinearCrossEntropy(20, 64, 300)
    M.forward(*args)
    assert torch.equal(L.backward(*args, accumulate_dw=1), M.backward(*args))
    assert torch.equal(L.dw, M.dw)
