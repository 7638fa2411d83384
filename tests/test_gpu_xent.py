"""The linear head's cross entropy against 64-bit arithmetic on the same inputs.

Tolerances, with u = 2^-24 (half an fp32 step) and h half a step of the element type.  A logit is an
fp32 sum of d exact products (bf16) or of d rounded ones (fp32), in an order that the matrix
instructions choose: off by at most (d + 1) u sum |x w|, and by 2 u |z| of the scale's product (ZE).
Exponentials have about one ulp (2 u) and the rounding of their argument (4 u |z - lse|); a row's sum
passes at most 64 additions in a lane, 2 across lanes, P / 16 partials of a thread and 16 of the
threads (each with two exponentials), P pieces of at least 32 columns.  The backward is held to the
forward's own lse; dz is rounded by h (bf16, up to 32 tokens: its two values leave h^2; more, with gradients of
their own: x with them by h too), sums over n terms have n u of the magnitudes.
"""
import math

import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.train import LinearCrossEntropy

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def half(dtype):
    return torch.finfo(dtype).eps / 2


def inputs(N, d, V, dtype, seed, ignored):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    w = (0.3 * r(V, d) / math.sqrt(d) * 3).to(DT[dtype])
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    x = (r(N, d) + 0.5 * w[labels].float()).to(DT[dtype])
    if ignored == "all":
        labels = torch.full_like(labels, -1)
    elif ignored:
        drop = torch.rand(N, generator=g, device="cuda") < ignored
        labels = torch.where(drop, torch.randint(-100, 0, (N,), generator=g, device="cuda"), labels)
    return dict(x=x, w=w, labels=labels.int(), dloss=torch.rand(N, generator=g, device="cuda") - 0.3)


def check(name, got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all(), name
    over = ((got - ref).abs() - tol).max().item() if ref.numel() else -1.0
    assert over <= 0, f"{name}: {over:.3e} past its bound"


def logits(t, scale):
    x, w = t["x"].double(), t["w"].double()
    z = scale * (x @ w.T)
    ze = abs(scale) * (x.shape[1] + 1) * U * (x.abs() @ w.abs().T) + 2 * U * z.abs()
    return z, ze


def check_forward(L, t, scale, z_coef):
    y = t["labels"].long()
    keep = y >= 0
    z, ze = logits(t, scale)
    V = z.shape[1]
    P = V // 32 + 2
    lse = torch.logsumexp(z, 1)
    far = (lse[:, None] - z).clamp(max=200).amax(1)
    e_lse = ze.amax(1) + (64 + 2 + P / 16 + 16 * 6 + 4) * U + 4 * U * far + 4 * U * lse.abs()
    zero = torch.zeros_like(lse)
    check("lse", L.lse, torch.where(keep, lse, zero), torch.where(keep, e_lse, zero))
    at = y.clamp(min=0)[:, None]
    zy, zye = z.gather(1, at)[:, 0], ze.gather(1, at)[:, 0]
    loss = lse - zy + z_coef * lse ** 2
    e = e_lse * (1 + 2 * abs(z_coef) * lse.abs()) + zye + 4 * U * (lse.abs() + zy.abs() + abs(z_coef) * lse ** 2)
    check("loss", L.loss, torch.where(keep, loss, zero), torch.where(keep, e, zero))
    n = int(keep.sum())
    assert L.total[1].item() == n
    ours = L.loss.double()
    assert abs(L.total[0].item() - ours.sum().item()) <= 2 * U * ours.abs().sum().item()


def check_backward(L, t, scale, z_coef, dloss, add=0.0):
    y = t["labels"].long()
    keep = y >= 0
    n = max(int(keep.sum()), 1)
    z, ze = logits(t, scale)
    N, V = z.shape
    lse = L.lse.double()[:, None]
    up = (torch.full((N,), 1.0 / n, device="cuda", dtype=torch.float64) if dloss is None else dloss.double())
    cf = torch.where(keep, up * scale, 0.0)[:, None]
    p = torch.exp(z - lse)
    zf = 1 + 2 * z_coef * lse
    one = torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], 1.0) * keep[:, None]
    dz = cf * (zf * p - one)
    h = half(L.dtype)
    # the relative error of p, the few products' and the difference's, then dz's own rounding
    e = cf.abs() * (zf * p).abs() * (ze + 4 * U * (z - lse).abs().clamp(max=200) + 10 * U) + 6 * U * cf.abs() * one
    hz = 2 * U if L.dtype != torch.bfloat16 else h * h if N <= 32 else h
    e = e + 6 * U * dz.abs()  # the factors that dz is taken out of and put back into: three products each
    e = e + hz * dz.abs() + 3 * U * dz.abs() + 1e-37
    x, w = t["x"].double(), t["w"].double()
    dx = dz @ w
    tol = e @ w.abs() + (V + 8) * U * (dz.abs() @ w.abs())
    check("dx", L.dx, dx, (tol + h * dx.abs()) * (1 + 2 * h) + 1e-37)
    xk = torch.where(keep[:, None], x, 0.0)
    dw = dz.T @ xk + add
    # (bf16, more than 32 tokens, gradients given: x comes with them, rounded by h beside dz)
    hx = h * (1 + h) if L.dtype == torch.bfloat16 and N > 32 and dloss is not None else 0.0
    tol = e.T @ xk.abs() + ((N + 8) * U + hx) * (dz.abs().T @ xk.abs()) + 2 * U * abs(add)
    check("dw", L.dw, dw, (tol + half(L.dw_dtype) * dw.abs()) * (1 + 2 * h) + 1e-37)
    assert (L.dx[~keep] == 0).all()


# (N, d, V, types, share that does not count): a token, fewer than a tile's and more; vocabularies of
# one word, around tiles' borders, of odd size; more tokens than one block counts; several pieces
CASES = [(1, 64, 1, "bf16 f32", 0), (1, 128, 5003, "bf16 f32", 0), (7, 64, 63, "bf16 f32", 0.4),
         (24, 192, 1000, "bf16 f32", 0), (33, 64, 257, "bf16 f32", 0.2), (100, 520, 130, "f32", 0.5),
         (65, 8, 100, "f32", 0), (128, 128, 300, "bf16 f32", "all"), (129, 64, 256, "bf16 f32", 0),
         (257, 192, 513, "bf16 f32", 0.5), (300, 1024, 2049, "bf16", 0), (1000, 256, 777, "bf16 f32", 0.97),
         (700, 320, 40, "bf16", 0.1), (500, 512, 9000, "bf16", 0.2), (1300, 1024, 3000, "bf16", 0),
         (1500, 640, 2500, "bf16", 0.3), (2100, 320, 5001, "bf16 f32", 0),
         (1200, 832, 20003, "bf16", 0.3), (60, 1088, 15001, "bf16", 0), (3000, 64, 12007, "f32", 0.1), (8193, 64, 1001, "bf16 f32", 0.3)]


@pytest.mark.gpu
@pytest.mark.parametrize("N,d,V,types,ignored", CASES)
def test_xent_matches_64_bits(gpu_lib, N, d, V, types, ignored):
    for dtype in types.split():
        for scale, z_coef, mean, low in ((1.0, 0.0, True, False), (-0.5, 1e-2, False, True)):
            print(f"[xent] N={N} d={d} V={V} {dtype} ignored={ignored} scale={scale}", flush=True)
            t = inputs(N, d, V, dtype, N + V, ignored)
            L = LinearCrossEntropy(N, d, V, dtype=DT[dtype], scale=scale, z_coef=z_coef,
                                   dw_dtype=DT[dtype] if low else torch.float32)
            for v in (L.loss, L.lse, L.total):
                v.fill_(float("nan"))
            loss = L.forward(t["x"], t["w"], t["labels"])
            assert loss is L.loss
            L.ws_fwd.fill_(255)  # nothing is kept between calls
            L.forward(t["x"], t["w"], t["labels"])
            check_forward(L, t, scale, z_coef)
            dloss = None if mean else t["dloss"]
            L.backward(t["x"], t["w"], t["labels"], dloss=dloss)
            for v in (L.dx, L.dw):
                v.fill_(float("nan"))
            L.ws_bwd.fill_(255)
            L.backward(t["x"], t["w"], t["labels"], dloss=dloss)
            check_backward(L, t, scale, z_coef, dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_xent_in_several_pieces(gpu_lib, dtype):
    """More logits' gradients than a piece holds."""
    N, d, V = (9001, 320, 20005) if dtype == "bf16" else (4500, 64, 40005)
    print(f"[xent pieces] {dtype}", flush=True)
    t = inputs(N, d, V, dtype, 5, 0.2)
    L = LinearCrossEntropy(N, d, V, dtype=DT[dtype])
    L.forward(t["x"], t["w"], t["labels"])
    check_forward(L, t, 1.0, 0.0)
    L.backward(t["x"], t["w"], t["labels"])
    check_backward(L, t, 1.0, 0.0, None)


@pytest.mark.gpu
def test_xent_of_weights_past_a_launchs_reach(gpu_lib):
    """More weights than one launch addresses: the forward in pieces of the vocabulary too."""
    N, d, V = 3, 16384, 33000
    print("[xent large weights]", flush=True)
    t = inputs(N, d, V, "bf16", 5, 0)
    L = LinearCrossEntropy(N, d, V, dw_dtype=torch.bfloat16)
    L.forward(t["x"], t["w"], t["labels"])
    check_forward(L, t, 1.0, 0.0)
    L.backward(t["x"], t["w"], t["labels"])
    check_backward(L, t, 1.0, 0.0, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,low", [("bf16", True), ("bf16", False), ("f32", False)])
def test_xent_adds_to_dw(gpu_lib, dtype, low):
    for N in (40, 300):
        t = inputs(N, 128, 521, dtype, 3, 0.2)
        L = LinearCrossEntropy(N, 128, 521, dtype=DT[dtype], dw_dtype=DT[dtype] if low else torch.float32)
        L.forward(t["x"], t["w"], t["labels"])
        L.backward(t["x"], t["w"], t["labels"], dloss=t["dloss"])
        L.dw.fill_(2.0)
        L.backward(t["x"], t["w"], t["labels"], dloss=t["dloss"], accumulate_dw=1)
        check_backward(L, t, 1.0, 0.0, t["dloss"], add=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [20, 200, 300])
def test_what_does_not_count_enters_nothing(gpu_lib, dtype, N):
    """Infinities and NaN in rows of tokens that do not count; their outputs are zeros."""
    t = inputs(N, 128, 300, dtype, 4, 0.5)
    gone = t["labels"] < 0
    L = LinearCrossEntropy(N, 128, 300, dtype=DT[dtype])
    run = lambda s: (L.forward(s["x"], s["w"], s["labels"]), L.backward(s["x"], s["w"], s["labels"]))
    run(t)
    ref = [v.clone() for v in (L.loss, L.lse, L.total, L.dx, L.dw)]
    s = dict(t, x=t["x"].clone())
    s["x"][gone] = float("nan")
    s["x"][gone.nonzero()[0, 0]] = float("inf")
    run(s)
    for a, b in zip((L.loss, L.lse, L.total, L.dx, L.dw), ref):
        assert torch.equal(a, b)
    assert (L.dx[gone] == 0).all() and (L.loss[gone] == 0).all() and (L.lse[gone] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("N", [20, 200, 300])
def test_a_label_that_is_no_word(gpu_lib, N):
    """V and more: the loss is NaN, and what the token enters in the backward."""
    V = 300
    t = inputs(N, 64, V, "bf16", 4, 0)
    ref = LinearCrossEntropy(N, 64, V)
    ref.forward(t["x"], t["w"], t["labels"])
    t["labels"][3], t["labels"][11] = V, 2 ** 31 - 1
    L = LinearCrossEntropy(N, 64, V)
    L.forward(t["x"], t["w"], t["labels"])
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[3] = bad[11] = True
    assert torch.isnan(L.loss[bad]).all() and torch.equal(L.loss[~bad], ref.loss[~bad])
    assert torch.equal(L.lse, ref.lse) and torch.isnan(L.total[0])
    L.backward(t["x"], t["w"], t["labels"])
    assert torch.isnan(L.dx[bad]).all() and torch.isfinite(L.dx[~bad].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,d,V", [(5, 64, 700), (200, 64, 700), (6000, 64, 5000)])
def test_nan_in_the_weights(gpu_lib, dtype, N, d, V):
    """Words whose rows are NaN, whole tiles of them and every one, make every counted token's loss NaN."""
    t = inputs(N, d, V, dtype, 9, 0.25)
    t["labels"][t["labels"] >= 0] = 3
    counts = t["labels"] >= 0
    L = LinearCrossEntropy(N, d, V, dtype=DT[dtype])
    for lo, hi in ((64, 577), (650, 651), (0, V)):
        w = t["w"].clone()
        w[lo:hi] = float("nan")
        L.forward(t["x"], w, t["labels"])
        assert torch.isnan(L.loss[counts]).all() and torch.isnan(L.lse[counts]).all(), (lo, hi)
        assert (L.loss[~counts] == 0).all() and torch.isnan(L.total[0])
        L.backward(t["x"], w, t["labels"])
        assert torch.isnan(L.dx[counts]).all() and (L.dx[~counts] == 0).all()
        assert torch.isnan(L.dw).all()  # (every word's gradient has those tokens' lse)


@pytest.mark.gpu
def test_no_tokens(gpu_lib):
    L = LinearCrossEntropy(0, 64, 100)
    x, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(100, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(0, dtype=torch.int32, device="cuda")
    L.forward(x, w, y)
    assert L.total.tolist() == [0.0, 0.0]
    L.backward(x, w, y)
    L.dw.fill_(4.0)
    L.backward(x, w, y, accumulate_dw=1)
    assert (L.dw == 4).all()
    L.backward(x, w, y)
    assert (L.dw == 0).all()


@pytest.mark.gpu
def test_xent_on_a_stream_and_in_a_graph(gpu_lib):
    """A captured step with other tokens, and other ones that count, at each replay."""
    N, d, V = 400, 128, 1500
    sets = [inputs(N, d, V, "bf16", s, p) for s, p in ((1, 0), (2, 0.4), (3, "all"))]
    w = sets[0]["w"]
    L = LinearCrossEntropy(N, d, V, z_coef=1e-3)

    def both(t, stream=None):
        L.forward(t["x"], w, t["labels"], stream=stream)
        L.backward(t["x"], w, t["labels"], stream=stream)

    def outs():
        torch.cuda.synchronize()
        return [v.clone() for v in (L.loss, L.lse, L.total, L.dx, L.dw)]

    refs = []
    for t in sets:
        both(t)
        refs.append(outs())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    both(sets[0], stream=s)
    assert all(torch.equal(a, b) for a, b in zip(outs(), refs[0]))
    live = {k: sets[0][k].clone() for k in ("x", "labels")}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(live)
    for i in (1, 0, 2, 1, 0):
        for k in live:
            live[k].copy_(sets[i][k])
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs(), refs[i])), i
        both(sets[i])
        assert all(torch.equal(a, b) for a, b in zip(outs(), refs[i])), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,d,V,lean", [(20, 64, 300, 30.0), (300, 128, 700, 6.0), (300, 128, 700, 40.0),
                                        (1300, 512, 4000, 12.0)])
def test_gradients_of_uneven_size(gpu_lib, dtype, N, d, V, lean):
    """Gradients from 1e-20 to 1e10, zeros, and no number where a token does not count; tokens that are
    nearly sure of their label, some of them of a probability that rounds to one."""
    t = inputs(N, d, V, dtype, 12, 0.2)
    y = t["labels"].long()
    lean = lean * torch.rand(N, 1, device="cuda")
    t["x"] = (t["x"].float() + lean * t["w"][y.clamp(min=0)].float()).to(DT[dtype])
    g = torch.randn(N, device="cuda") * 10.0 ** torch.linspace(-20, 10, N, device="cuda")
    g[::7] = 0.0
    g[y < 0] = float("nan")
    for scale, z_coef in ((1.0, 0.0), (1.5, 1e-2)):
        L = LinearCrossEntropy(N, d, V, dtype=DT[dtype], scale=scale, z_coef=z_coef)
        L.forward(t["x"], t["w"], t["labels"])
        L.backward(t["x"], t["w"], t["labels"], dloss=g)
        check_backward(L, t, scale, z_coef, torch.where(y < 0, 0.0, g))


@pytest.mark.gpu
@pytest.mark.parametrize("N", [20, 300])
def test_given_gradients_in_a_graph(gpu_lib, N):
    """A captured backward with other gradients, tokens and labels at each replay."""
    d, V = 128, 900
    sets = [inputs(N, d, V, "bf16", s, p) for s, p in ((1, 0), (2, 0.4), (3, 0))]
    w, L = sets[0]["w"], LinearCrossEntropy(N, d, V)

    def both(t):
        L.forward(t["x"], w, t["labels"])
        L.backward(t["x"], w, t["labels"], dloss=t["dloss"])

    def outs():
        torch.cuda.synchronize()
        return [v.clone() for v in (L.loss, L.total, L.dx, L.dw)]

    refs = []
    for t in sets:
        both(t)
        refs.append(outs())
    live = {k: sets[0][k].clone() for k in ("x", "labels", "dloss")}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(live)
    for i in (1, 0, 2, 1):
        for k in live:
            live[k].copy_(sets[i][k])
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs(), refs[i])), i
        both(sets[2 - i])
        assert all(torch.equal(a, b) for a, b in zip(outs(), refs[2 - i])), i


@pytest.mark.gpu
def test_two_heads_at_once(gpu_lib):
    """Two objects on two streams, their launches beside each other."""
    N, d, V = 700, 256, 3000
    sets = [inputs(N, d, V, "bf16", s, 0.2) for s in (1, 2)]
    heads = [LinearCrossEntropy(N, d, V) for _ in sets]
    outs = lambda: [v.clone() for L in heads for v in (L.loss, L.lse, L.total, L.dx, L.dw)]
    for L, t in zip(heads, sets):
        L.forward(t["x"], t["w"], t["labels"])
        L.backward(t["x"], t["w"], t["labels"])
    torch.cuda.synchronize()
    ref, streams = outs(), [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for call in ("forward", "backward"):
            for L, t, s in zip(heads, sets, streams):
                getattr(L, call)(t["x"], t["w"], t["labels"], stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs(), ref))


@pytest.mark.gpu
def test_xent_gradients_against_differences(gpu_lib):
    """<dx, ex> + <dw, ew> against a central difference in 64 bits of the weighted losses."""
    N, d, V, scale, zc = 9, 64, 70, 0.7, 0.02
    t = inputs(N, d, V, "f32", 6, 0.2)
    L = LinearCrossEntropy(N, d, V, dtype=torch.float32, scale=scale, z_coef=zc)
    L.forward(t["x"], t["w"], t["labels"])
    L.backward(t["x"], t["w"], t["labels"], dloss=t["dloss"])
    y = t["labels"].long()

    def value(x, w):
        z = scale * x @ w.T
        lse = torch.logsumexp(z, 1)
        loss = lse - z.gather(1, y.clamp(min=0)[:, None])[:, 0] + zc * lse ** 2
        return (torch.where(y >= 0, loss, 0.0) * t["dloss"].double()).sum().item()

    X, W = t["x"].double(), t["w"].double()
    g = torch.Generator(device="cuda").manual_seed(8)
    ex, ew = (torch.randn(v.shape, generator=g, device="cuda").double() for v in (X, W))
    e = 1e-5
    num = (value(X + e * ex, W + e * ew) - value(X - e * ex, W - e * ew)) / (2 * e)
    parts = L.dx.double() * ex, L.dw.double() * ew
    ours, mag = sum(v.sum().item() for v in parts), sum(v.abs().sum().item() for v in parts)
    assert abs(num - ours) <= 1e-5 * mag


@pytest.mark.gpu
def test_xent_refuses(gpu_lib):
    L = LinearCrossEntropy(4, 64, 10)
    x, w = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(10, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args in ((x.float(), w, y), (x[:3], w, y), (x, w[:9], y), (x, w, y.long()), (x, w.t(), y),
                 (x.cpu(), w, y), (x, w, y[:3])):
        with pytest.raises(ValueError):
            L.forward(*args)
    with pytest.raises(ValueError):
        L.backward(x, w, y, dloss=torch.ones(4, dtype=torch.float64, device="cuda"))
    for kw in (dict(dtype=torch.float16), dict(dw_dtype=torch.float16),
               dict(dtype=torch.float32, dw_dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            LinearCrossEntropy(4, 64, 10, **kw)
    with pytest.raises(B.MoeError):  # bf16: a width of 64s
        M = LinearCrossEntropy(4, 72, 10)
        M.forward(torch.ones(4, 72, dtype=torch.bfloat16, device="cuda"),
                  torch.ones(10, 72, dtype=torch.bfloat16, device="cuda"), y)


def test_c_entry_points_refuse():
    import ctypes as C
    L, p = B.lib(), 1 << 12  # (an address that is never read)
    good = dict(dtype=B.MOE_BF16, N=4, d=64, V=10, scale=1.0, x=p, w=p, labels=p, loss=p, lse=p, total=p,
                dx=p, dw=p, ws=p, ws_bytes=1 << 40)
    arg, unsupported = -1, -2
    both = [(dict(dtype=4), unsupported), (dict(N=-1), arg), (dict(V=0), arg), (dict(d=0), arg),
            (dict(dtype=B.MOE_F32, N=1 << 23), unsupported), (dict(d=72), unsupported), (dict(d=1 << 17), unsupported),
            (dict(N=1 << 22, d=512), unsupported), (dict(N=1 << 23), unsupported),
            (dict(dtype=B.MOE_F32, N=1 << 22, d=512), unsupported),
            (dict(V=1 << 30), unsupported), (dict(dtype=B.MOE_F32, d=12), unsupported),
            (dict(scale=math.inf), arg), (dict(scale=0.0), arg), (dict(z_coef=math.nan), arg), (dict(x=None), arg),
            (dict(w=None), arg), (dict(labels=None), arg), (dict(lse=None), arg),
            (dict(x=p + 8), unsupported), (dict(w=p + 2), unsupported), (dict(ws=None), arg),
            (dict(ws_bytes=100), arg), (dict(ws=p + 16), unsupported)]
    fwd = [(dict(loss=None), arg), (dict(total=None), arg)]
    bwd = [(dict(dx=None), arg), (dict(dw=None), arg), (dict(dw_dtype=2), unsupported),
           (dict(dtype=B.MOE_F32, dw_dtype=B.MOE_BF16), unsupported), (dict(dw=p + 4), unsupported)]
    for fn, cases in (("moe_xent_fwd", both + fwd), ("moe_xent_bwd", both + bwd)):
        for kw, want in cases:
            assert getattr(L, fn)(C.byref(B.moe_xent(**dict(good, **kw))), None) == want, (fn, kw)
            assert B.moe_last_error()
        assert getattr(L, fn)(None, None) == arg
    assert L.moe_xent_fwd_workspace_size(C.byref(B.moe_xent(**dict(good, d=72)))) == 0
