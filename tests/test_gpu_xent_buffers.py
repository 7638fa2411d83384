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


@pytest.mark.gpu
def test_a_captured_backward_adds_at_every_replay(gpu_lib):
    """Behind an earlier call, whose dw it adds to; as an object's first backward it is refused, as what
    makes dw zeros would be replayed with it."""
    args = small()
    ref = LinearCrossEntropy(20, 64, 300)
    ref.forward(*args)
    ref.backward(*args)
    L, M = (LinearCrossEntropy(20, 64, 300) for _ in range(2))
    L.forward(*args)
    M.forward(*args)
    M.backward(*args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(ValueError):
            L.backward(*args, accumulate_dw=1)
        M.backward(*args, accumulate_dw=1)
    assert L.dx is None and L.dw is None and L.ws_bwd is None
    want = ref.dw.clone()
    for _ in range(4):
        g.replay()
        ref.backward(*args, accumulate_dw=1)
        torch.cuda.synchronize()
        assert torch.equal(M.dw, ref.dw) and not torch.equal(M.dw, want)
        want = M.dw.clone()
        L.backward(*args, accumulate_dw=1)  # (eager work between the replays)
    # (L's dw: zeros, and what its four calls between the replays added)
    four = LinearCrossEntropy(20, 64, 300)
    four.forward(*args)
    for i in range(4):
        four.backward(*args, accumulate_dw=int(i > 0))
    assert torch.equal(L.dw, four.dw)


@pytest.mark.gpu
def test_a_captured_first_backward_overwrites(gpu_lib):
    """Without adding to dw the first backward may be captured, and another one behind it adds."""
    args = small()
    ref, L = (LinearCrossEntropy(20, 64, 300) for _ in range(2))
    for X in (ref, L):
        X.forward(*args)
    ref.backward(*args)
    ref.backward(*args, accumulate_dw=1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.backward(*args)
        L.backward(*args, accumulate_dw=1)
    for _ in range(3):
        L.dw.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.dw, ref.dw) and torch.equal(L.dx, ref.dx)
