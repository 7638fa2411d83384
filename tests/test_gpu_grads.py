"""The norm of many gradients, clipping, and AdamW over many tensors.

Sums of squares are held in fp64, so the norm is off by its rounding to fp32 (2^-24, with the
fp64 sum's n 2^-53 below a thousandth of that); the scale by that and its own rounding.  What is
multiplied by the scale is exact in the same order of fp32 operations."""
import math

import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.train import AdamW, GradClipper

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
# sizes around the ends of vectors and chunks; more tensors than a launch's table holds
SIZES = {
    "one": [1], "odd": [1, 3, 7, 8, 9, 16383, 16384, 16385, 32771, 5], "empty": [0, 5, 0],
    "large": [3_000_001, 40, 1 << 20], "many": [1 + (i * 37) % 611 for i in range(300)],
    "tables": [9] * 173 + [4097] + [7] * 98 + [8191] + [3] * 200,
}


def make(sizes, seed, types=(F32, BF), std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * std * (1 + i % 5)).to(types[i % len(types)])
            for i, n in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(SIZES))
def test_norm_and_clip(gpu_lib, kind):
    grads = make(SIZES[kind], 3)
    ref = norm_of(grads)
    for max_norm in (0.37 * ref, 2 * ref, math.inf):
        print(f"[grads] {kind} max_norm={max_norm}", flush=True)
        out = [torch.full_like(g, float("nan")) for g in grads]
        n = GradClipper(grads, max_norm, out=out).clip()
        got, scale = n.tolist()
        assert abs(got - ref) <= 1.001 * U * ref
        want = min(1.0, max_norm / ref)
        assert abs(scale - want) <= 2.01 * U * want and (scale == 1.0) == (max_norm > ref)
        for g, o in zip(grads, out):
            assert torch.equal(o, (g.float() * n[1]).to(g.dtype))
        # in place, and the same bits again
        own = [g.clone() for g in grads]
        assert torch.equal(GradClipper(own, max_norm).clip(), n)
        assert all(torch.equal(a, b) for a, b in zip(own, out))


@pytest.mark.gpu
def test_a_tensor_past_32_bit_offsets(gpu_lib):
    """2^31 + 7 bf16 values among small ones."""
    n = (1 << 31) + 7
    print("[grads] large", flush=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    big = torch.empty(n, dtype=BF, device="cuda").normal_(generator=g)
    small = make([5, 70], 1)
    out = [torch.empty_like(big)] + [torch.empty_like(s) for s in small]
    norm = GradClipper([big] + small, 3.0, out=out).clip()
    ref = math.sqrt(sum(float((c.double() ** 2).sum()) for c in big.split(1 << 28)) + norm_of(small) ** 2)
    assert abs(norm[0].item() - ref) <= 1.001 * U * ref
    for a, b in zip([big[-4096:], big[:4096], big[(1 << 31) - 9: (1 << 31) + 3]] + small,
                    [out[0][-4096:], out[0][:4096], out[0][(1 << 31) - 9: (1 << 31) + 3]] + out[1:]):
        assert torch.equal(b, (a.float() * norm[1]).to(a.dtype))


@pytest.mark.gpu
def test_unaligned_gradients(gpu_lib):
    """Pieces of one buffer that start at any value."""
    flat = {F32: make([5000], 1)[0], BF: make([5000], 2, (BF,))[0]}
    cuts = [0, 1, 4, 9, 1030, 1031, 2049, 4999, 5000]
    grads = [f[a:b] for f in flat.values() for a, b in zip(cuts, cuts[1:])]
    ref = norm_of(grads)
    out = [torch.empty(g.numel() + 3, dtype=g.dtype, device="cuda")[i % 4: i % 4 + g.numel()] for i, g in enumerate(grads)]
    n = GradClipper(grads, 1.0, out=out).clip()
    assert abs(n[0].item() - ref) <= 1.001 * U * ref
    for g, o in zip(grads, out):
        assert torch.equal(o, (g.float() * n[1]).to(g.dtype))
    before = {t: f.clone() for t, f in flat.items()}
    GradClipper([g for g in grads[::2]], 1.0).clip()
    for f, g in zip(flat.values(), (0, 1)):
        for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
            if (i + g * (len(cuts) - 1)) % 2:  # not in the list: as it was
                assert torch.equal(f[a:b], before[f.dtype][a:b])


@pytest.mark.gpu
def test_sizes_of_values(gpu_lib):
    """Squares that leave fp32's range at either end; zeros; infinities and NaN."""
    big, tiny = torch.full((1000,), 1e30, device="cuda"), torch.full((1000,), 1e-30, device="cuda")
    for g in (big, tiny):
        n = GradClipper([g], 1.0, out=[torch.empty_like(g)]).clip()
        ref = float(g[0]) * math.sqrt(1000)
        assert abs(n[0].item() - ref) <= 1.001 * U * ref
    z = torch.zeros(1000, device="cuda")
    assert GradClipper([z], 1.0).clip().tolist() == [0.0, 1.0]
    for bad in (math.inf, math.nan):
        g = make([100, 50], 5)
        g[1][7] = bad
        keep, out = [v.clone() for v in g], [torch.zeros_like(v) for v in g]
        n = GradClipper(g, 1e-3, out=out).clip().tolist()
        assert math.isnan(n[1]) and not math.isfinite(n[0])
        same = lambda a, b: all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, b))
        assert same(out, keep)
        GradClipper(g, 1e-3).clip()
        assert same(g, keep)


def state(sizes, seed, types):
    grads = make(sizes, seed, types)
    theta = make(sizes, seed + 1, (F32,))
    m = make(sizes, seed + 2, (F32,), std=0.1)
    v = [x.square() for x in make(sizes, seed + 3, (F32,), std=0.1)]
    return theta, grads, m, v, [t.bfloat16() for t in theta]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["odd", "empty", "large", "many", "tables"])
@pytest.mark.parametrize("clipped", [True, False])
def test_adamw_steps_is_adamw_step_of_clipped_gradients(gpu_lib, kind, clipped):
    sizes = SIZES[kind]
    theta, grads, m, v, low = state(sizes, 7, (F32, BF))
    low = [x if i % 3 else None for i, x in enumerate(low)]
    decay, rate = [0.1 * (i % 2) for i in range(len(sizes))], [1.0 + 0.25 * (i % 4) for i in range(len(sizes))]
    ref = norm_of(grads)
    copy = lambda lst: [None if x is None else x.clone() for x in lst]
    want = [copy(x) for x in (theta, m, v, low)]
    opt = AdamW(theta, grads, m, v, theta_bf16=low, max_norm=0.5 * ref if clipped else None,
                weight_decay=decay, lr_scale=rate)
    for t in (1, 2, 9):
        norm = opt.step(t, 1e-3)
        assert (norm is None) == (not clipped)
        for i, n in enumerate(sizes):
            g = grads[i].float() * (norm[1] if clipped else 1.0)
            lr = (torch.tensor(1e-3) * torch.tensor(rate[i])).item()
            B.moe_adamw_step(want[0][i], g, want[1][i], want[2][i], n, t, lr, weight_decay=decay[i],
                             theta_bf16=want[3][i])
        for got, ours in zip(want, (theta, m, v, low)):
            assert all(a is None or torch.equal(a, b) for a, b in zip(got, ours)), t


@pytest.mark.gpu
def test_no_step_on_a_norm_that_is_not_finite(gpu_lib):
    theta, grads, m, v, low = state([300, 9000], 1, (F32, BF))
    grads[1][5] = math.nan
    keep = [[x.clone() for x in lst] for lst in (theta, m, v, low)]
    n = AdamW(theta, grads, m, v, theta_bf16=low, max_norm=1.0).step(1, 1e-3)
    assert math.isnan(n[0].item())
    assert all(torch.equal(a, b) for old, new in zip(keep, (theta, m, v, low)) for a, b in zip(old, new))


@pytest.mark.gpu
def test_on_a_stream_and_in_a_graph(gpu_lib):
    """A captured step, replayed with other gradients between eager ones."""
    def fresh(seed):
        return state([5000, 77, 20001], seed, (F32, BF))
    sets = [make([5000, 77, 20001], s) for s in (21, 22)]
    live = [g.clone() for g in sets[0]]
    theta, _, m, v, low = fresh(1)
    opt = AdamW(theta, live, m, v, theta_bf16=low, max_norm=1.0)
    t2, _, m2, v2, low2 = fresh(1)
    eager = [AdamW(t2, g, m2, v2, theta_bf16=low2, max_norm=1.0) for g in sets]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    opt.step(3, 1e-3, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    eager[0].step(3, 1e-3)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.step(3, 1e-3)
    for i in (0, 1, 0, 1):
        for a, b in zip(live, sets[i]):
            a.copy_(b)
        g.replay()
        n = eager[i].step(3, 1e-3)
        torch.cuda.synchronize()
        assert torch.equal(opt.norm, n)
        for a, b in zip(theta + m + v + low, t2 + m2 + v2 + low2):
            assert torch.equal(a, b)


def test_refusals_without_a_gpu():
    f, b = torch.zeros(8), torch.zeros(8, dtype=BF)
    for args, kw in ((([], 1.0), {}), (([f], 0.0), {}), (([f], -1.0), {}), (([f], math.nan), {}),
                     (([f.double()], 1.0), {}), (([f, 3], 1.0), {}), (([f.view(4, 2).t()], 1.0), {}),
                     (([f], 1.0), dict(out=[b])), (([f], 1.0), dict(out=[f, f])),
                     (([f, f], 1.0), {}), (([f, f[4:]], 1.0), {}),
                     (([f[:4], f[4:]], 1.0), dict(out=[f[4:], torch.zeros(4)])),
                     (([f[:4], f[4:]], 1.0), dict(out=[torch.zeros(4), f[2:6]]))):
        with pytest.raises(ValueError):
            GradClipper(*args, **kw)
    for theta, grads, kw in (([b], [b], {}), ([f], [f[:4]], {}), ([f], [f, f], {}), ([f], [f.double()], {}),
                             ([f], [f], dict(m=[f])), ([f], [f], dict(theta_bf16=[f])),
                             ([f], [torch.ones(8)], dict(weight_decay=[0.1, 0.1])),
                             ([f, f], [torch.ones(8), torch.ones(8)], {}), ([f], [f], {}),
                             ([f], [torch.ones(8)], dict(m=[f], v=[torch.ones(8)]))):
        with pytest.raises(ValueError):
            AdamW(theta, grads, **kw)


def test_c_entry_points_refuse():
    L, p = B.lib(), 1 << 12  # (an address that is never read)
    grads = lambda *g: (B.moe_grad * len(g))(*[B.moe_grad(*x) for x in g])
    arg, unsupported = -1, -2
    norm = lambda g, n, mx=1.0, out=p, ws=p, size=1 << 20: L.moe_grad_norm(g, n, mx, out, ws, size, None)
    ok = grads((p, p, 8, B.MOE_F32))
    for got, want in ((norm(ok, -1), arg), (norm(None, 1), arg), (norm(ok, 1, mx=0.0), arg),
                      (norm(ok, 1, mx=math.nan), arg), (norm(ok, 1, out=None), arg),
                      (norm(ok, 1, size=4), arg), (norm(ok, 1, ws=None), arg),
                      (norm(ok, 1, ws=p + 4), unsupported), (norm(ok, 1, out=p + 2), unsupported),
                      (norm(grads((None, p, 8, 0)), 1), arg), (norm(grads((p, p, 8, 5)), 1), unsupported),
                      (norm(grads((p + 2, p, 8, 0)), 1), unsupported),
                      (norm(grads((p, p, 1 << 44, 0)), 1), unsupported),
                      (L.moe_grad_clip(ok, 1, None, None), arg),
                      (L.moe_grad_clip(grads((p, None, 8, 0)), 1, p, None), arg),
                      (L.moe_grad_clip(grads((p, p + 1, 8, 1)), 1, p, None), unsupported)):
        assert got == want, B.moe_last_error()
    t = lambda **kw: (B.moe_adamw_tensor * 1)(B.moe_adamw_tensor(**{**dict(
        theta=p, grad=p, m=p, v=p, n=8, lr_scale=1.0), **kw}))
    step = lambda a, n=1, s=1, b1=0.9, b2=0.95, eps=1e-8, norm=None: L.moe_adamw_steps(
        a, n, s, 1e-3, b1, b2, eps, norm, None)
    for got, want in ((step(t(), n=-1), arg), (step(None), arg), (step(t(), s=0), arg),
                      (step(t(), b1=1.0), arg),
                      (step(t(), eps=-1.0), arg), (step(t(m=None)), arg), (step(t(grad=p + 4)), unsupported),
                      (step(t(theta_bf16=p + 8)), unsupported), (step(t(grad_dtype=3)), unsupported),
                      (step(t(n=1 << 43)), unsupported), (step(t(), norm=p + 1), unsupported)):
        assert got == want, B.moe_last_error()
