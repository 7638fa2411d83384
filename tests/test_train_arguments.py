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
