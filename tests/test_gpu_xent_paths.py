"""Paths of the linear head's cross entropy that only certain sizes reach, against 64-bit arithmetic, with the
tolerances of test_gpu_xent: several pieces of the vocabulary together with the tokens' own gradients,
sums and left-out tokens; dW added to in large tiles; several tiles of few k-steps to a block."""
import math

import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.train import LinearCrossEntropy

from .test_gpu_xent import DT, check_backward, check_forward, half, inputs


def launches(call):
    """{name: launches} of a call."""
    B.moe_timing_enable(256)
    try:
        call()
        torch.cuda.synchronize()
        return {k: v[0] for k, v in B.moe_timing_collect().items()}
    finally:
        B.moe_timing_enable(0)


def step(N, d, V, dtype, ignored=0.2, given=False, add=None, low=False, scale=1.0, z_coef=0.0, seed=5):
    """A forward and a backward checked; the names of both calls' launches."""
    print(f"[xent paths] N={N} d={d} V={V} {dtype} given={given} add={add} low={low}", flush=True)
    t = inputs(N, d, V, dtype, seed, ignored)
    dloss = t["dloss"] if given else None
    L = LinearCrossEntropy(N, d, V, dtype=DT[dtype], scale=scale, z_coef=z_coef,
                           dw_dtype=DT[dtype] if low else torch.float32)
    fwd = launches(lambda: L.forward(t["x"], t["w"], t["labels"]))
    check_forward(L, t, scale, z_coef)
    L.backward(t["x"], t["w"], t["labels"], dloss=dloss)
    for v in (L.dx, L.dw):
        v.fill_(float("nan"))
    L.ws_bwd.fill_(255)
    if add is not None:
        L.dw.fill_(add)
    bwd = launches(lambda: L.backward(t["x"], t["w"], t["labels"], dloss=dloss,
                                      accumulate_dw=int(add is not None)))
    check_backward(L, t, scale, z_coef, dloss, add=add or 0.0)
    return fwd, bwd


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("add", [None, 2.0])
@pytest.mark.parametrize("dtype,low", [("bf16", False), ("bf16", True), ("f32", False)])
def test_pieces_of_the_vocabulary(gpu_lib, dtype, low, given, add):
    """dz of all words is more than a piece: dx is summed over pieces, dW written or added to piece by piece, and the
    rows, coefficients and factors that the first launch makes are used again by each."""
    N, d, V = (9001, 512, 20005) if dtype == "bf16" else (4500, 64, 40005)
    fwd, bwd = step(N, d, V, dtype, given=given, add=add, low=low, z_coef=1e-3, scale=0.75)
    name = "gemm_xe_dx_dw" + ("" if dtype == "bf16" else "_tile")
    assert bwd[name] >= 2, bwd


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [False, True])
def test_pieces_of_the_forward_with_tokens_left_out(gpu_lib, dtype, given):
    """More weights than a launch addresses, of tokens that are copied together first: each piece's partial sums
    and label's logits are those of the copied rows."""
    fwd, bwd = step(300, 16384, 33000, dtype, ignored=0.3, given=given)
    assert fwd["xent_rows"] == 1
    assert sum(n for k, n in fwd.items() if k.startswith("gemm_xe_lse")) == 2, fwd


@pytest.mark.gpu
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_large_tiles_add_to_dw(gpu_lib, low, given):
    """fp32 and bf16 values of dW, some of whose tiles reach past the last word and the last column."""
    fwd, bwd = step(2500, 1088, 12007, "bf16", given=given, add=-3.0, low=low)
    assert "gemm_xe_dx_dw" in bwd, bwd


@pytest.mark.gpu
@pytest.mark.parametrize("N,d,V", [(6000, 64, 5000), (9000, 128, 9001), (5000, 192, 7003)])
def test_several_tiles_of_few_k_steps(gpu_lib, N, d, V):
    """Blocks of the large tiles that take one after another, of one to three k-steps: the next one's first
    loads under the epilogue, in rings that they fill in part."""
    fwd, bwd = step(N, d, V, "bf16", given=True)
    assert "gemm_xe_lse" in fwd and "gemm_xe_dz" in bwd, (fwd, bwd)
    # more tiles of 256 x 256 than CUs
    assert math.ceil(0.7 * N / 256) * math.ceil(V / 256) > torch.cuda.get_device_properties(0).multi_processor_count


# ---- tokens' own gradients: the label's entry of dz is left out of its rounding

def folded(N=600, d=128, V=2048):
    """Inputs whose gradients g make the label's entry of dz, g (p - 1), lie nearly half a step of bf16 above
    one; in 64 bits that entry, the other words' and the words' rows."""
    g = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g)
    x, w = r(N, d).bfloat16(), (r(V, d) / math.sqrt(d)).bfloat16()
    y = torch.randint(0, V, (N,), generator=g)
    z = x.double() @ w.double().T
    p = torch.softmax(z, 1)
    q = p.gather(1, y[:, None])[:, 0] - 1
    dloss = ((1 + 0.98 * 2.0 ** -8) / q).float()
    dz = dloss.double()[:, None] * p
    others = dz.scatter(1, y[:, None], 0.0)
    return dict(x=x, w=w, y=y, dloss=dloss, label=dloss.double() * q, others=others)


def dx_of(t, label):
    """dx of a label's entry, with the other words' as they are."""
    dz = t["others"].scatter(1, t["y"][:, None], label[:, None])
    return dz @ t["w"].double()


def norm_bound(t, dx):
    """On the norm of dx's error where the label's entry is not rounded.  A rounding to bf16 is off by at most h
    of the value, and its square by at most h^2 / 3 in the mean over the values within a step: so dx's own
    rounding by h^2 / 3 of |dx|^2, and the other words' entries, whose roundings are of different words, by h^2 / 3
    of the sum of |dz_tv w_v|^2.  Five per cent more for the mean over 76800 values, whose spread is below 1 %."""
    h = half(torch.bfloat16)
    squares = dx.pow(2).sum() + (t["others"] ** 2 @ t["w"].double().pow(2).sum(1)).sum()
    return 1.05 * h / math.sqrt(3) * math.sqrt(squares)


def test_the_bound_tells_a_rounded_label():
    """The oracle with its outputs rounded is within the bound, and with the label's entry rounded too is not."""
    t = folded()
    dx = dx_of(t, t["label"])
    off = lambda label: (dx_of(t, label).bfloat16().double() - dx).norm().item()
    bound = norm_bound(t, dx)
    assert off(t["label"]) < bound
    assert off(t["label"].bfloat16().double()) > 1.5 * bound


@pytest.mark.gpu
def test_a_labels_entry_is_not_rounded(gpu_lib):
    t = folded()
    N, d = t["x"].shape
    V = t["w"].shape[0]
    x, w, y = t["x"].cuda(), t["w"].cuda(), t["y"].int().cuda()
    L = LinearCrossEntropy(N, d, V)
    L.forward(x, w, y)
    L.backward(x, w, y, dloss=t["dloss"].cuda())
    dx = dx_of(t, t["label"])
    assert (L.dx.cpu().double() - dx).norm().item() <= norm_bound(t, dx)
