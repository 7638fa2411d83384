"""Layer norm, forward and backward, against 64-bit arithmetic on the same inputs.

Tolerances, with u = 2^-24 (half an fp32 step) and h half a step of the element type: a
sum over a row is a chain of at most 16 additions per lane, 6 across a wave and 16 across
waves, so its error is at most 40 u times the sum of magnitudes (SUM); sums over T <= 3001
rows pass at most 6 rows of a wave, 4 waves, 32 + 16 partials (COLS = 64).  The products
and differences around them add a few u of the magnitudes that enter, counted below.
"""
import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.layer import LayerNorm, PreNormMoELayer

U = 2.0 ** -24
SUM, COLS = 40, 64
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# (T, d): one wave, four and sixteen per row; ragged widths; the ends of each range
SHAPES = [(1, 8), (1, 2048), (3, 520), (7, 4104), (2, 16384), (5, 16376), (1023, 72), (1024, 1024),
          (1500, 1032), (1025, 2048), (1030, 4096), (3001, 520)]


def half(dtype):
    return torch.finfo(DT[dtype]).eps / 2


def inputs(T, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    x = (r(T, d) * r(d).mul(0.3).exp() + r(T, 1)).to(DT[dtype]).cuda()
    return dict(x=x, w=(1 + 0.2 * r(d)).cuda(), b=(0.2 * r(d)).cuda(),
                dy=r(T, d).to(DT[dtype]).cuda(), dres=r(T, d).to(DT[dtype]).cuda())


def check(name, got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all(), name
    over = ((got - ref).abs() - tol).max().item() if ref.numel() else -1.0
    assert over <= 0, f"{name}: {over:.3e} past its bound"


def check_forward(x, w, b, eps, y, mean, rstd, h):
    X, W = x.double(), w.double()
    mu = X.mean(1, keepdim=True)
    var = ((X - mu) ** 2).mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    A = X.abs().amax(1, keepdim=True)
    xh = (X - mu) * r
    ref = xh * W + (0 if b is None else b.double())
    # the mean's error moves every element; var's relative error is SUM u and that of its
    # terms (two roundings of x - mu, at most 2 u A each, relative to 1 / r)
    d_mu, d_r = SUM * U * A, (SUM / 2 + 4) * U + 4 * U * A * r
    check("mean", mean, mu[:, 0], d_mu[:, 0])
    check("rstd", rstd, r[:, 0], (r * d_r)[:, 0] + 2 * d_mu[:, 0] ** 2 * r[:, 0] ** 3)
    tol = W.abs() * (xh.abs() * (d_r + 3 * U) + r * (d_mu + 2 * U * A)) + 3 * U * ref.abs() + h * ref.abs()
    if b is not None:
        tol = tol + 2 * U * b.double().abs()
    check("y", y, ref, tol * (1 + h) + 1e-300)


def check_backward(dy, x, w, mean, rstd, dres, dx, dw, db, h, dw0=0.0, db0=0.0):
    X, G0, W = x.double(), dy.double(), w.double()
    r = rstd.double()[:, None]
    xh = (X - mean.double()[:, None]) * r
    g = G0 * W
    m0, m1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    a0, a1 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
    ref = r * (g - m0 - xh * m1)
    tol = r * (SUM + 8) * U * (g.abs() + a0 + xh.abs() * a1)
    if dres is not None:
        ref = ref + dres.double()
        tol = tol + 2 * U * dres.double().abs()
    check("dx", dx, ref, (tol + 2 * U * ref.abs() + h * ref.abs()) * (1 + h) + 1e-300)
    t = G0 * xh
    check("dw", dw, t.sum(0) + dw0, (COLS + 4) * U * t.abs().sum(0) + 2 * U * abs(dw0) + 1e-300)
    if db is not None:
        check("db", db, G0.sum(0) + db0, (COLS + 4) * U * G0.abs().sum(0) + 2 * U * abs(db0) + 1e-300)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_norm_matches_64_bits(gpu_lib, T, d, dtype):
    print(f"[norm] T={T} d={d} {dtype}", flush=True)
    for bias, res in ((True, False), (False, True)):
        t = inputs(T, d, dtype, seed=T + d)
        N = LayerNorm(T, d, dtype=DT[dtype], bias=bias)
        b = t["b"] if bias else None
        N.forward(t["x"], t["w"], b)
        check_forward(t["x"], t["w"], b, 1e-5, N.y, N.mean, N.rstd, half(dtype))
        dres = t["dres"] if res else None
        N.backward(t["dy"], t["x"], t["w"], dres=dres)
        check_backward(t["dy"], t["x"], t["w"], N.mean, N.rstd, dres, N.dx, N.dw, N.db, half(dtype))
        assert (N.db is None) == (not bias)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", [(4096, 8, "bf16"), (4097, 520, "bf16"), (4099, 1024, "bf16"),
                                       (4100, 2040, "bf16"), (4096, 256, "f32"), (5003, 264, "f32"),
                                       (4098, 520, "f32"), (4101, 1024, "f32")])
def test_norm_a_row_per_wave(gpu_lib, T, d, dtype):
    """Many rows: one wave each (at most 4 rows of a wave, 4 waves, 512 partials by 64 shares)."""
    test_norm_matches_64_bits(gpu_lib, T, d, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", [(300, 4104, "bf16"), (601, 8192, "bf16"), (1100, 16384, "bf16"),
                                       (299, 4104, "f32"), (700, 16376, "f32")])
def test_norm_sixteen_waves_take_several_rows(gpu_lib, T, d, dtype):
    """More rows than blocks where a row is a block's sixteen waves' (at most 5 rows of a block, one
    addition each, 275 partials)."""
    test_norm_matches_64_bits(gpu_lib, T, d, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [((1 << 26) + 5, 8), ((1 << 24) + 3, 2056), ((1 << 22) + 1, 8200)])
def test_norm_more_rows_than_a_grid(gpu_lib, T, d):
    """Rows of one, four and sixteen waves, more of them than a launch's 2^32 threads hold, in
    place: every row is written, and those around the launches' borders are right."""
    if torch.cuda.mem_get_info()[0] < 2 * T * d + 12 * T + (4 << 30):
        pytest.skip("not enough free memory")
    print(f"[norm] T={T} d={d}", flush=True)
    t = inputs(64, d, "bf16", seed=T + d)
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    x[: T // 64 * 64].view(-1, 64, d)[:] = t["x"]
    x[T // 64 * 64:] = t["x"][: T % 64]
    mean, rstd = torch.full((2, T), float("nan"), device="cuda")
    B.moe_layernorm_fwd(x, t["w"], t["b"], B.MOE_BF16, T, d, 1e-5, x, mean, rstd)
    check_forward(t["x"], t["w"], t["b"], 1e-5, x[:64], mean[:64], rstd[:64], half("bf16"))
    for v in (mean, rstd):  # the same rows again and again
        assert torch.equal(v[: T // 64 * 64].view(-1, 64), v[:64].expand(T // 64, 64))
        assert torch.equal(v[T // 64 * 64:], v[: T % 64])
    step = max(1, (1 << 28) // (64 * d))  # (in parts: a comparison of all needs as many bytes again)
    for lo in range(0, T // 64, step):
        hi = min(T // 64, lo + step)
        assert (x[64 * lo:64 * hi].view(-1, 64, d) == x[:64]).all(), lo
    assert torch.equal(x[T // 64 * 64:], x[: T % 64])
    del x, mean, rstd
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_equal_and_huge(gpu_lib, dtype):
    """Rows of one value whose multiple by rstd overflows: x - mean is zero, and the lanes past
    the row's end (x zero there, the mean not) must not make it NaN.  The sums of 8 terms
    are exact for x (a power of two); for g they take at most 9 additions and two products."""
    x = torch.full((6, 8), 2.0 ** 120, dtype=DT[dtype], device="cuda")
    t = inputs(6, 8, dtype, seed=3)
    N = LayerNorm(6, 8, dtype=DT[dtype])
    N.forward(x, t["w"], t["b"])
    assert (N.mean == 2.0 ** 120).all()
    N.backward(t["dy"], x, t["w"])
    g = t["dy"].double() * t["w"].double()
    ref = N.rstd.double()[:, None] * (g - g.mean(1, keepdim=True))
    tol = 16 * U * N.rstd.double()[:, None] * (g.abs() + g.abs().mean(1, keepdim=True))
    check("dx", N.dx, ref, (tol + half(dtype) * ref.abs()) * (1 + half(dtype)))
    assert (N.dw == 0).all() and torch.isfinite(N.db).all()


@pytest.mark.gpu
def test_norm_first_backward_in_a_graph(gpu_lib):
    """Its first backward captured, adding to dw: every replay adds."""
    t = inputs(40, 256, "f32", seed=8)
    M = LayerNorm(40, 256, dtype=torch.float32)
    M.forward(t["x"], t["w"], t["b"])
    M.backward(t["dy"], t["x"], t["w"])
    N = LayerNorm(40, 256, dtype=torch.float32)
    N.forward(t["x"], t["w"], t["b"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        N.backward(t["dy"], t["x"], t["w"], accumulate_dw=1)
    for i in range(1, 5):
        g.replay()
        torch.cuda.synchronize()
        # (i sums of equal parts: one rounding each)
        assert ((N.dw - i * M.dw).abs() <= i * i * U * M.dw.abs()).all()
        assert ((N.db - i * M.db).abs() <= i * i * U * M.db.abs()).all()
        assert torch.equal(N.dx, M.dx)


@pytest.mark.gpu
def test_norm_against_differences(gpu_lib):
    """The gradients of L = sum(y * dy) against central differences of the 64-bit forward: step
    e = 1e-5 leaves a relative error of order e^2, far under the 1e-4 allowed to fp32."""
    T, d, e = 3, 64, 1e-5
    t = inputs(T, d, "f32", seed=3)
    N = LayerNorm(T, d, dtype=torch.float32)
    N.forward(t["x"], t["w"], t["b"])
    N.backward(t["dy"], t["x"], t["w"])
    X, W, Bi, G = (t[k].double().cpu() for k in ("x", "w", "b", "dy"))

    def loss(X, W, Bi):
        mu = X.mean(1, keepdim=True)
        return ((X - mu) / (((X - mu) ** 2).mean(1, keepdim=True) + 1e-5).sqrt() * W + Bi).mul(G).sum()

    def diff(v, i):
        hi, lo = ([a.clone() for a in (X, W, Bi)] for _ in range(2))
        hi[v].view(-1)[i] += e
        lo[v].view(-1)[i] -= e
        return ((loss(*hi) - loss(*lo)) / (2 * e)).item()

    for v, got in ((0, N.dx), (1, N.dw), (2, N.db)):
        got = got.cpu().view(-1)
        for i in range(0, got.numel(), 7):
            ref = diff(v, i)
            assert abs(got[i].item() - ref) <= 1e-4 * max(1.0, abs(ref)), (v, i)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_hard_rows(gpu_lib, dtype):
    """Rows far from zero, of equal values, of zeros, of tiny and of large values; a row of NaN
    or infinity stays in its own row."""
    T, d = 9, 200
    t = inputs(T, d, dtype, seed=5)
    x = t["x"].float()
    x[0] += 3e4
    x[1] = 7.0
    x[2] = 0.0
    x[3] *= 1e-18
    x[4] *= 1e15
    x = x.to(DT[dtype]).contiguous()
    N = LayerNorm(T, d, dtype=DT[dtype])
    N.forward(x, t["w"], t["b"])
    check_forward(x, t["w"], t["b"], 1e-5, N.y, N.mean, N.rstd, half(dtype))
    ok = [0, 1, 2, 3, 5, 6, 7, 8]
    N.backward(t["dy"], x, t["w"])
    check_backward(t["dy"], x, t["w"], N.mean, N.rstd, None, N.dx, N.dw, N.db, half(dtype))
    clean = N.y[ok].clone()
    x[4, 3], x[4, 150] = float("nan"), float("inf")
    N.forward(x, t["w"], t["b"])
    assert torch.equal(N.y[ok], clean) and N.y[4].isnan().all()


@pytest.mark.gpu
def test_norm_zero_rows(gpu_lib):
    """No rows: nothing to write but dw and db, zeros or left as they are."""
    N = LayerNorm(0, 64, dtype=torch.float32)
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    N.forward(e, w, w)
    N.backward(e, e, w)
    N.dw.fill_(3.0)
    N.backward(e, e, w, accumulate_dw=1)
    assert (N.dw == 3).all() and (N.db == 0).all()
    N.backward(e, e, w)
    assert (N.dw == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", [(37, 1032, "bf16"), (1100, 512, "f32")])
def test_norm_bounds_aliases_and_sums(gpu_lib, T, d, dtype):
    """Rows behind the last stay as they are; y in x's place, dx in dy's or dres's; dw and db
    added to; the same bits on every call."""
    t = inputs(T, d, dtype, seed=11)
    pad = lambda v: torch.cat([v, torch.full((2, d), 7.0, device="cuda", dtype=v.dtype)])
    N = LayerNorm(T, d, dtype=DT[dtype])
    N.forward(t["x"], t["w"], t["b"])
    N.backward(t["dy"], t["x"], t["w"], dres=t["dres"])
    y, dx, dw, db = N.y.clone(), N.dx.clone(), N.dw.clone(), N.db.clone()
    mean, rstd = torch.full((2, T + 1), 7.0, device="cuda")
    buf = pad(t["x"])
    B.moe_layernorm_fwd(buf, t["w"], t["b"], N.dt, T, d, 1e-5, buf, mean, rstd)
    assert torch.equal(buf[:T], y) and (buf[T:] == 7).all() and mean[T] == 7 and rstd[T] == 7
    for name in ("dy", "dres"):
        at = {k: pad(t[k]) for k in ("dy", "dres")}
        B.moe_layernorm_bwd(at["dy"], t["x"], t["w"], mean, rstd, N.dt, T, d, at["dres"], at[name],
                            N.dw, N.db, 0, N.ws, N.ws_bytes)
        assert torch.equal(at[name][:T], dx) and (at[name][T:] == 7).all()
        assert torch.equal(N.dw, dw) and torch.equal(N.db, db)
    N.backward(t["dy"], t["x"], t["w"], accumulate_dw=1)
    assert torch.equal(N.dw, dw + dw) and torch.equal(N.db, db + db)


@pytest.mark.gpu
def test_norm_stream_and_graph(gpu_lib):
    """A stream of the caller's, and a captured pass replayed with new inputs."""
    T, d = 300, 768
    a, b = (inputs(T, d, "bf16", seed=s) for s in (1, 2))
    N = LayerNorm(T, d)

    def both(t):
        N.forward(t["x"], t["w"], t["b"])
        N.backward(t["dy"], t["x"], t["w"])

    def outs():
        torch.cuda.synchronize()
        return [v.clone() for v in (N.y, N.dx, N.dw, N.db)]

    both(a)
    ref_a = outs()
    both(b)
    ref_b = outs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    N.forward(a["x"], a["w"], a["b"], stream=s)
    N.backward(a["dy"], a["x"], a["w"], stream=s)
    assert all(torch.equal(u, v) for u, v in zip(outs(), ref_a))
    live = {k: v.clone() for k, v in a.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(live)
    for t, ref in ((a, ref_a), (b, ref_b), (a, ref_a), (b, ref_b)):
        for k, v in t.items():
            live[k].copy_(v)
        g.replay()
        assert all(torch.equal(u, v) for u, v in zip(outs(), ref))
        both(t)
        assert all(torch.equal(u, v) for u, v in zip(outs(), ref))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pre_norm_layer_is_norm_then_layer(gpu_lib, dtype):
    """PreNormMoELayer: the layer on the norm's output, and back with the residual's gradient."""
    from .parity_helpers import dev
    from .test_gpu_parity import synth_inputs
    inp = synth_inputs(130, 128, 12, 3, 128, [0, 3, 5, 8], dtype, seed=7, shared_hidden=64)
    dt = DT[dtype]
    w = {n: dev(inp[n], dt) for n in ("w_router", "w_gate_up", "w_down", "shared_gate_up", "shared_down")}
    x, dy = dev(inp["x"], dt), dev(inp["dy"], dt)
    nw, nb = torch.rand(128, device="cuda") + 0.5, torch.randn(128, device="cuda")
    P = PreNormMoELayer(130, 128, 12, 3, 128, inp["resident"], dtype=dt, n_shared_hidden=64)
    y = P.forward(x, nw, nb, **w).clone()
    dx = P.backward(dy, x, nw, **w).clone()
    check_forward(x, nw, nb, 1e-5, P.norm.y, P.norm.mean, P.norm.rstd, half(dtype))
    assert torch.equal(y, P.layer.forward(P.norm.y, **w))
    check_backward(P.layer.dx, x, nw, P.norm.mean, P.norm.rstd, dy, dx, P.norm.dw, P.norm.db, half(dtype))


def test_norm_refusals():
    """Bad sizes, pointers and workspaces are refused on the host."""
    if torch.cuda.device_count() > 0:
        pytest.skip("host-only rejection test: runs where no GPU is visible")
    L, p = B.lib(), 256  # a fake, never dereferenced address

    def fwd(x=p, w=p, b=p, dt=B.MOE_BF16, T=4, d=64, eps=1e-5, y=p, m=p, r=p):
        return L.moe_layernorm_fwd(x, w, b, dt, T, d, eps, y, m, r, None)

    assert fwd(dt=7) == -2 and fwd(d=60) == -2 and fwd(d=16392) == -2 and fwd(x=p + 2) == -2
    assert fwd(T=-1) == -1 and fwd(d=0) == -1 and fwd(w=None) == -1 and fwd(x=None) == -1
    assert fwd(eps=float("nan")) == -1 and fwd(eps=-1.0) == -1 and fwd(y=None) == -1 and fwd(r=None) == -1
    need = B.moe_layernorm_bwd_workspace_size(4, 64, B.MOE_BF16)
    assert need >= 2 * 64 * 4 and B.moe_layernorm_bwd_workspace_size(-1, 64, 0) == 0
    assert B.moe_layernorm_bwd_workspace_size(4, 2 ** 31 - 1, 0) == 0  # (sizes that are refused)
    assert B.moe_layernorm_bwd_workspace_size(4, 60, 0) == 0 and fwd(T=1 << 30) == -2

    def bwd(dy=p, x=p, w=p, m=p, r=p, dt=B.MOE_BF16, T=4, d=64, res=None, dx=p, dw=p, db=p, ws=p, n=need):
        return L.moe_layernorm_bwd(dy, x, w, m, r, dt, T, d, res, dx, dw, db, 0, ws, n, None)

    assert bwd(n=need - 1) == -1 and "workspace" in B.moe_last_error()
    assert bwd(ws=None) == -1 and bwd(dw=None) == -1 and bwd(m=None) == -1 and bwd(dx=None) == -1
    assert bwd(ws=p + 8) == -2 and bwd(res=p + 8) == -2 and bwd(d=12) == -2 and bwd(dt=3) == -2


def test_norm_class_checks():
    N = LayerNorm(4, 64, dtype=torch.float32, device="cpu")
    x, w = torch.zeros(4, 64), torch.zeros(64)
    for args in ((x.T, w, w), (x.bfloat16(), w, w), (x, w[:8], w), (x, w, None), (None, w, w)):
        with pytest.raises(ValueError):
            N.forward(*args)
    with pytest.raises(ValueError):
        LayerNorm(4, 64, bias=False, dtype=torch.float32, device="cpu").forward(x, w, w)
    with pytest.raises(ValueError):
        LayerNorm(4, 64, dtype=torch.float16, device="cpu")
