"""What the training step's classes accept and refuse where they are made, on tensors of the CPU."""
import math

import pytest
import torch

from paper_2606_19025_amd.train import AdamW

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("max_norm", [None, 1.0, math.inf])
def test_a_gradient_given_to_several_parameters(max_norm):
    """The norm is measured and written nowhere near the gradients, so they may share memory."""
    g = torch.ones(8)
    opt = AdamW([torch.zeros(8), torch.zeros(8)], [g, g], max_norm=max_norm)
    assert (opt.norm is None) == (max_norm is None)
    AdamW([torch.zeros(8), torch.zeros(4)], [g, g[4:]], max_norm=max_norm)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_gradient_given_to_several_parameters_counts_as_often(gpu_lib, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    grad = torch.randn(5000, generator=g, device="cuda").to(dtype)
    make = lambda: [torch.full((5000,), v, device="cuda") for v in (1.0, -2.0)]
    shared, apart = make(), make()
    n = AdamW(shared, [grad, grad], max_norm=1.0).step(1, 1e-3)
    want = AdamW(apart, [grad, grad.clone()], max_norm=1.0).step(1, 1e-3)
    assert torch.equal(n, want) and all(torch.equal(a, b) for a, b in zip(shared, apart))
    # the norm's rounding to fp32 over its fp64 sum
    ref = math.sqrt(2 * float((grad.double() ** 2).sum()))
    assert abs(n[0].item() - ref) <= 1.001 * 2.0 ** -24 * ref


def test_misaligned_tensors_are_refused_at_construction():
    """All that the optimiser reads and writes is 16-byte aligned; a list that is not is no list for it."""
    at = lambda dtype, k: torch.zeros(16, dtype=dtype)[k:k + 8]
    good = lambda: dict(theta=[at(F32, 0), at(F32, 4)], grads=[at(F32, 8), at(BF, 8)],
                        m=[at(F32, 4), at(F32, 0)], v=[at(F32, 0), at(F32, 0)], theta_bf16=[None, at(BF, 0)])
    AdamW(**good())
    for name, dtype, k in (("theta", F32, 1), ("theta", F32, 2), ("grads", F32, 3), ("grads", BF, 4),
                           ("grads", BF, 1), ("m", F32, 1), ("v", F32, 6), ("theta_bf16", BF, 2)):
        for max_norm in (None, 1.0):
            bad = good()
            bad[name][1] = at(dtype, k)
            with pytest.raises(ValueError):
                AdamW(**bad, max_norm=max_norm)
    empty = torch.zeros(16)[1:1]  # (no values: nothing is read)
    assert empty.numel() == 0
    AdamW([empty], [empty])
