"""The norms and the residual sum around a block, against 64-bit arithmetic on the same inputs.

Tolerances, with u = 2^-24 (half an fp32 step) and h half a step of the element type.  Sums over a
row or over rows as in the layer norm's tests: SUM u and COLS u of the sums of magnitudes.  The
backward passes G, with a bound of its own, through the gate and the post norm: its bound is
carried along by the formulas' magnitudes, beside the new roundings.
"""
import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.layer import BlockNorm, LayerNorm, PeriNormMoELayer

from .test_gpu_norm import COLS, DT, SUM, U, check, check_forward, half

# (T, d): one to sixteen waves a row, several rows for each; ragged widths; the ends of the ranges
SHAPES = [(600, 4104), (300, 8208), (700, 600), (2100, 1024), (530, 2056), (1, 8), (1, 2048), (3, 520), (7, 4104), (2, 16384), (5, 8200), (1023, 72), (300, 1032),
          (4099, 512), (4100, 264), (4096, 8), (1030, 4096), (3001, 520), (20001, 264), (13001, 520),
          (9001, 1032), (3001, 2056), (2001, 4168)]
# (post, pre, gate, bias)
FORMS = [(True, True, None, True), (True, True, "channel", True), (True, True, "token", False),
         (False, True, "channel", False), (False, True, "token", True), (True, False, None, True),
         (True, False, "channel", True), (True, False, "token", True)]


def inputs(T, d, dtype, seed, gate):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    act = lambda t: t.to(DT[dtype]).cuda()
    t = dict(x=act(r(T, d) * r(d).mul(0.3).exp() + r(T, 1)), f=act(0.5 * r(T, d) + 0.2 * r(T, 1)),
             du=act(r(T, d)), dres=act(r(T, d)))
    for n in ("post", "pre"):
        t[n + "_weight"], t[n + "_bias"] = (1 + 0.2 * r(d)).cuda(), (0.2 * r(d)).cuda()
    t["gate"] = None if gate is None else (0.5 + 0.3 * r(d if gate == "channel" else T)).cuda()
    return t


def weights(t, post, pre, bias):
    return dict(post_weight=t["post_weight"] if post else None,
                post_bias=t["post_bias"] if post and bias else None, gate=t["gate"],
                pre_weight=t["pre_weight"] if pre else None), (t["pre_bias"] if pre and bias else None)


def factor(scale, gate, kind):
    if kind is None:
        return torch.full((1, 1), scale, dtype=torch.float64, device="cuda")
    return scale * (gate.double()[:, None] if kind == "token" else gate.double()[None])


def check_block_forward(K, t, w, pre_bias, kind, scale, h, eps=1e-5):
    F, X = t["f"].double(), t["x"].double()
    n, tol = F, torch.zeros_like(F)
    if K.post:
        W = w["post_weight"].double()
        mu = F.mean(1, keepdim=True)
        r = (((F - mu) ** 2).mean(1, keepdim=True) + eps) ** -0.5
        A, xh = F.abs().amax(1, keepdim=True), (F - mu) * r
        d_mu, d_r = SUM * U * A, (SUM / 2 + 4) * U + 4 * U * A * r
        check("post_mean", K.post_mean, mu[:, 0], d_mu[:, 0])
        check("post_rstd", K.post_rstd, r[:, 0], (r * d_r)[:, 0] + 2 * d_mu[:, 0] ** 2 * r[:, 0] ** 3)
        n = xh * W
        tol = W.abs() * (xh.abs() * (d_r + 3 * U) + r * (d_mu + 2 * U * A))
        if w["post_bias"] is not None:
            n = n + w["post_bias"].double()
            tol = tol + 2 * U * (n.abs() + w["post_bias"].double().abs())
    g = factor(scale, t["gate"], kind)
    ref = X + g * n
    tol = g.abs() * (tol + 4 * U * n.abs()) + 2 * U * ref.abs()
    check("x", K.x, ref, (tol + h * ref.abs()) * (1 + h) + 1e-300)
    if K.pre:  # of x' as it was rounded
        check_forward(K.x, w["pre_weight"], pre_bias, eps, K.u, K.pre_mean, K.pre_rstd, h)


def check_block_backward(K, t, w, kind, scale, h, du, dres, x, add=0.0):
    F = t["f"].double()
    G = torch.zeros_like(F) if dres is None else dres.double()
    tol = 2 * U * G.abs()
    if K.pre:
        r = K.pre_rstd.double()[:, None]
        xh = (x.double() - K.pre_mean.double()[:, None]) * r
        D = du.double()
        q = D * w["pre_weight"].double()
        m0, m1 = q.mean(1, keepdim=True), (q * xh).mean(1, keepdim=True)
        a0, a1 = q.abs().mean(1, keepdim=True), (q * xh).abs().mean(1, keepdim=True)
        G = G + r * (q - m0 - xh * m1)
        tol = tol + r * (SUM + 8) * U * (q.abs() + a0 + xh.abs() * a1) + 2 * U * G.abs()
        s = D * xh
        check("d_pre_weight", K.d_pre_weight, s.sum(0) + add,
              (COLS + 4) * U * s.abs().sum(0) + 2 * U * abs(add) + 1e-300)
        if K.d_pre_bias is not None:
            check("d_pre_bias", K.d_pre_bias, D.sum(0) + add,
                  (COLS + 4) * U * D.abs().sum(0) + 2 * U * abs(add) + 1e-300)
    check("dx", K.dx, G, (tol + h * G.abs()) * (1 + h) + 1e-300)
    g = factor(scale, t["gate"], kind)
    fh, n, aff = F, F, torch.ones_like(F)
    if K.post:
        r2 = K.post_rstd.double()[:, None]
        fh = (F - K.post_mean.double()[:, None]) * r2
        aff = w["post_weight"].double().expand_as(F)
        b = w["post_bias"].double() if w["post_bias"] is not None else torch.zeros_like(F)
        n = fh * aff + b
        dn, d_dn = g * G, g.abs() * (tol + 4 * U * G.abs())
        for name, out, v, e in (("d_post_weight", K.d_post_weight, dn * fh, d_dn * fh.abs()),
                                ("d_post_bias", K.d_post_bias, dn, d_dn)):
            if out is not None:
                check(name, out, v.sum(0) + add, e.sum(0) + (COLS + 8) * U * v.abs().sum(0)
                      + 2 * U * abs(add) + 1e-300)
        q, e = dn * aff, d_dn * aff.abs() + 2 * U * (dn * aff).abs()
        mean = lambda v: v.mean(1, keepdim=True)
        ref = r2 * (q - mean(q) - fh * mean(q * fh))
        bound = r2 * (e + mean(e) + fh.abs() * mean(e * fh.abs())
                      + (SUM + 8) * U * (q.abs() + mean(q.abs()) + fh.abs() * mean((q * fh).abs())))
    else:
        ref = g * G
        bound = g.abs() * (tol + 4 * U * G.abs())
    check("df", K.df, ref, (bound + h * ref.abs()) * (1 + h) + 1e-300)
    if kind is not None:
        # sums of scale G n: of n's two terms by themselves
        mag = G.abs() * ((fh * aff).abs() + (n - fh * aff).abs()) * abs(scale)
        err = tol * n.abs() * abs(scale)
        dim = 1 if kind == "token" else 0
        more = 0.0 if kind == "token" else add
        check("d_gate", K.d_gate, (scale * G * n).sum(dim) + more,
              err.sum(dim) + (max(SUM, COLS) + 10) * U * mag.sum(dim) + 2 * U * abs(more) + 1e-300)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_block_norm_matches_64_bits(gpu_lib, T, d, dtype):
    h = half(dtype)
    for i, (post, pre, kind, bias) in enumerate(FORMS):
        print(f"[block] T={T} d={d} {dtype} post={post} pre={pre} gate={kind} bias={bias}", flush=True)
        t = inputs(T, d, dtype, T + d + i, kind)
        w, pre_bias = weights(t, post, pre, bias)
        K = BlockNorm(T, d, dtype=DT[dtype], post=post, pre=pre, gate=kind, bias=bias, scale=0.7)
        x, u = K.forward(t["x"], t["f"], **w, pre_bias=pre_bias)
        assert x is K.x and u is K.u and (u is None) == (not pre)
        check_block_forward(K, t, w, pre_bias, kind, 0.7, h)
        du = t["du"] if pre else None
        dres = t["dres"] if i % 2 or not pre else None
        K.backward(du, t["f"], **w, dres=dres)
        check_block_backward(K, t, w, kind, 0.7, h, du, dres, K.x)


@pytest.mark.gpu
def test_block_norm_adds_where_asked(gpu_lib):
    for kind in (None, "channel", "token"):
        t = inputs(70, 264, "bf16", 5, kind)
        w, pre_bias = weights(t, True, True, True)
        K = BlockNorm(70, 264, gate=kind)
        K.forward(t["x"], t["f"], **w, pre_bias=pre_bias)
        K.backward(t["du"], t["f"], **w, dres=t["dres"])
        for v in (K.d_post_weight, K.d_post_bias, K.d_pre_weight, K.d_pre_bias, K.d_gate):
            if v is not None:
                v.fill_(3.0)
        K.backward(t["du"], t["f"], **w, dres=t["dres"], accumulate=1)
        check_block_backward(K, t, w, kind, 1.0, half("bf16"), t["du"], t["dres"], K.x, add=3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(33, 520), (1100, 2048), (600, 8192), (300, 12288)])
def test_block_norm_in_place(gpu_lib, T, d, dtype):
    """x_out in x, dx in dres or du, df in f; also where a row's arrays are fetched rounds ahead."""
    t = inputs(T, d, dtype, 9, "channel")
    w, pre_bias = weights(t, True, True, True)
    K = BlockNorm(T, d, dtype=DT[dtype], gate="channel")
    K.forward(t["x"], t["f"], **w, pre_bias=pre_bias)
    K.backward(t["du"], t["f"], **w, dres=t["dres"])
    ref = [v.clone() for v in (K.x, K.u, K.dx, K.df, K.d_gate)]
    for target in ("dres", "du"):
        L = BlockNorm(T, d, dtype=DT[dtype], gate="channel")
        s = {k: v.clone() for k, v in t.items()}
        L.x = s["x"]
        L.forward(s["x"], s["f"], **w, pre_bias=pre_bias)
        L.backward(s["du"], s["f"], **w, dres=s["dres"])  # (makes its buffers)
        L.dx, L.df = s[target], s["f"]
        L._args.dx, L._args.df = L.dx.data_ptr(), L.df.data_ptr()
        L.backward(s["du"], s["f"], **w, dres=s["dres"])
        assert all(torch.equal(a, b) for a, b in zip((L.x, L.u, L.dx, L.df, L.d_gate), ref)), target


@pytest.mark.gpu
def test_rows_past_32_bit_offsets(gpu_lib):
    """The last rows of arrays of over 2^31 values: bit for bit those of the rows alone (of as many
    rows as take a wave each, so that sums run in the same order)."""
    T, d, n = (1 << 31) // 2048 + 100, 2048, 4160
    print("[block] large", flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda").normal_(generator=g)
    x, f, du = r(T, d), r(T, d), r(T, d)
    w = dict(post_weight=r(d, dt=torch.float32), post_bias=r(d, dt=torch.float32),
             gate=r(T, dt=torch.float32), pre_weight=r(d, dt=torch.float32))
    K, S = BlockNorm(T, d, gate="token"), BlockNorm(n, d, gate="token")
    K.forward(x, f, **w, pre_bias=w["pre_weight"])
    K.backward(du, f, **w, dres=x)
    last = lambda t: t[T - n:].contiguous()
    ws = dict(w, gate=last(w["gate"]))
    S.forward(last(x), last(f), **ws, pre_bias=w["pre_weight"])
    S.backward(last(du), last(f), **ws, dres=last(x))
    for a, b in ((K.x, S.x), (K.u, S.u), (K.dx, S.dx), (K.df, S.df), (K.d_gate, S.d_gate)):
        assert torch.equal(last(a), b)
    # sums over T rows: at most T / 512 of a group, two groups, 256 partials by 64 shares
    ref, mag = (sum(v.double().sum(0) for v in f_(du).split(1 << 16)) for f_ in (lambda v: v, torch.abs))
    assert ((K.d_pre_bias.double() - ref).abs() <= (T / 512 + 20) * U * mag).all()


@pytest.mark.gpu
def test_block_norm_of_no_rows(gpu_lib):
    w = {k: torch.ones(64, device="cuda") for k in ("post_weight", "post_bias", "gate", "pre_weight")}
    K = BlockNorm(0, 64, gate="channel")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    K.forward(e, e, **w, pre_bias=w["post_bias"])
    for v in (K.d_post_weight, K.d_post_bias, K.d_pre_weight, K.d_pre_bias, K.d_gate):
        v.fill_(5.0)
    K.backward(e, e, **w, accumulate=1)
    assert (K.d_gate == 5).all() and (K.d_post_weight == 5).all()
    K.backward(e, e, **w)
    for v in (K.d_post_weight, K.d_post_bias, K.d_pre_weight, K.d_pre_bias, K.d_gate):
        assert (v == 0).all()


@pytest.mark.gpu
def test_block_norm_on_a_stream_and_in_a_graph(gpu_lib):
    T, d = 300, 768
    a, b = (inputs(T, d, "bf16", s, "token") for s in (1, 2))
    K = BlockNorm(T, d, gate="token", scale=0.5)
    wa, pre_bias = weights(a, True, True, True)
    keep = {k: v for k, v in wa.items() if k != "gate"}

    def both(t, stream=None):
        K.forward(t["x"], t["f"], **keep, gate=t["gate"], pre_bias=pre_bias, stream=stream)
        K.backward(t["du"], t["f"], **keep, gate=t["gate"], dres=t["dres"], stream=stream)

    def outs():
        torch.cuda.synchronize()
        return [v.clone() for v in (K.x, K.u, K.dx, K.df, K.d_gate, K.d_post_weight, K.d_post_bias,
                                    K.d_pre_weight, K.d_pre_bias)]

    both(a)
    ref_a = outs()
    both(b)
    ref_b = outs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    both(a, stream=s)
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
def test_block_norm_gradients_against_differences(gpu_lib):
    """<dx, ex> + <df, ef> + <d_gate, eg> against a central difference of <x', cx> + <u, cu>,
    evaluated in 64 bits: the formulas themselves (fp32 gradients, so the bound is the
    difference's own h^2 error and fp32 sums, far below 1e-4 of the magnitudes)."""
    T, d = 5, 64
    for post, pre, kind in ((True, True, "channel"), (True, True, "token"), (False, True, None)):
        t = inputs(T, d, "f32", 11, kind)
        w, pre_bias = weights(t, post, pre, True)
        K = BlockNorm(T, d, dtype=torch.float32, post=post, pre=pre, gate=kind, scale=0.8)
        K.forward(t["x"], t["f"], **w, pre_bias=pre_bias)
        K.backward(t["du"], t["f"], **w, dres=t["dres"])

        def value(x, f, gate):
            norm = lambda v, a, c: ((v - v.mean(1, keepdim=True)) * (v.var(1, unbiased=False, keepdim=True) + 1e-5) ** -0.5) * a.double() + c.double()
            n = norm(f, w["post_weight"], w["post_bias"]) if post else f
            x = x + (0.8 if kind is None else 0.8 * (gate[:, None] if kind == "token" else gate)) * n
            return ((x * t["dres"].double()).sum() + (norm(x, w["pre_weight"], pre_bias) * t["du"].double()).sum()).item()

        X, F = t["x"].double(), t["f"].double()
        g0 = torch.zeros(1, device="cuda").double() if kind is None else t["gate"].double()
        gen = torch.Generator().manual_seed(3)
        e = [torch.randn(v.shape, generator=gen).double().cuda() for v in (X, F, g0)]
        step = 1e-5
        num = (value(X + step * e[0], F + step * e[1], g0 + step * e[2])
               - value(X - step * e[0], F - step * e[1], g0 - step * e[2])) / (2 * step)
        parts = [K.dx.double() * e[0], K.df.double() * e[1]]
        if kind is not None:
            parts.append(K.d_gate.double() * e[2])
        ours = sum(v.sum().item() for v in parts)
        mag = sum(v.abs().sum().item() for v in parts)
        assert abs(num - ours) <= 1e-4 * mag, (post, pre, kind, num, ours)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peri_norm_blocks_chain(gpu_lib, dtype):
    """Two Peri-LN blocks behind a first norm: each the layer and the block norm on the other's
    outputs, and back."""
    from .parity_helpers import dev
    from .test_gpu_parity import synth_inputs
    T, d = 130, 128
    inp = synth_inputs(T, d, 12, 3, 128, [0, 3, 5, 8], dtype, seed=7, shared_hidden=64)
    dt, h = DT[dtype], half(dtype)
    lw = {n: dev(inp[n], dt) for n in ("w_router", "w_gate_up", "w_down", "shared_gate_up", "shared_down")}
    x, dy = dev(inp["x"], dt), dev(inp["dy"], dt)
    ones, zeros = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    t = [inputs(T, d, dtype, s, "channel") for s in (1, 2)]
    nw = [dict(zip(("post_weight", "post_bias", "gate", "pre_weight"), (q["post_weight"], q["post_bias"],
               q["gate"], q["pre_weight"])), pre_bias=q["pre_bias"]) for q in t]
    nw[1].update(pre_weight=None, pre_bias=None)
    first = LayerNorm(T, d, dtype=dt)
    P = [PeriNormMoELayer(T, d, 12, 3, 128, inp["resident"], dtype=dt, n_shared_hidden=64, gate="channel",
                          scale=0.5, pre=i == 0) for i in range(2)]
    u0 = first.forward(x, ones, zeros)
    x1, u1 = P[0].forward(x, u0, nw[0], **lw)
    x2, u2 = P[1].forward(x1, u1, nw[1], **lw)
    assert u2 is None
    for p, xin, uin, i in ((P[0], x, u0, 0), (P[1], x1, u1, 1)):
        y = p.layer.y.clone()
        assert torch.equal(y, p.layer.forward(uin, **lw))
        w = {k: v for k, v in nw[i].items() if k != "pre_bias"}
        check_block_forward(p.norm, dict(t[i], x=xin, f=y), w, nw[i]["pre_bias"], "channel", 0.5, h)
    du1, dx1 = P[1].backward(None, dy, u1, nw[1], **lw)
    du0, dx0 = P[0].backward(du1, dx1, u0, nw[0], **lw)
    for p, du, dres, xo, i in ((P[1], None, dy, x2, 1), (P[0], du1, dx1, x1, 0)):
        w = {k: v for k, v in nw[i].items() if k != "pre_bias"}
        check_block_backward(p.norm, dict(t[i], f=p.layer.y), w, "channel", 0.5, h, du, dres, xo)
    df = P[0].norm.df
    assert torch.equal(du0, P[0].layer.backward(df, u0, **lw))


@pytest.mark.gpu
def test_block_norm_refuses(gpu_lib):
    v = torch.ones(64, device="cuda")
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    K = BlockNorm(4, 64)
    full = dict(post_weight=v, post_bias=v, pre_weight=v, pre_bias=v)
    bad = [dict(full, post_weight=None), dict(full, pre_bias=None), dict(full, gate=v),
           dict(full, post_weight=v.bfloat16()), dict(full, pre_weight=torch.ones(128, device="cuda")[::2])]
    for w in bad:
        with pytest.raises(ValueError):
            K.forward(x, x, **w)
    with pytest.raises(ValueError):
        K.forward(x.float(), x, **full)
    with pytest.raises(ValueError):
        K.forward(x, x[:3], **full)
    with pytest.raises(ValueError):
        K.backward(None, x, post_weight=v, post_bias=v, pre_weight=v)
    L = BlockNorm(4, 64, pre=False)
    with pytest.raises(ValueError):
        L.backward(x, x, post_weight=v, post_bias=v, dres=x)
    with pytest.raises(ValueError):
        L.backward(None, x, post_weight=v, post_bias=v)


def test_block_norm_arguments_are_checked_on_the_host():
    """The C entry points' own checks: no launch, so they hold without a GPU."""
    import ctypes as C
    p = 1 << 12  # (an address that is never read)
    good = dict(dtype=B.MOE_BF16, T=4, d=64, gate_kind=0, scale=1.0, eps=1e-5, x=p, f=p, x_out=p, u=p,
                post_weight=p, pre_weight=p, post_mean=p, post_rstd=p, pre_mean=p, pre_rstd=p)
    L = B.lib()
    call = lambda fn, **kw: getattr(L, fn)(C.byref(B.moe_block_norm(**dict(good, **kw))), None)
    arg, unsupported = -1, -2
    fwd = [(dict(T=-1), arg), (dict(d=0), arg), (dict(d=60), unsupported), (dict(d=16392), unsupported),
           (dict(T=1 << 30), unsupported), (dict(dtype=7), unsupported), (dict(gate_kind=3), arg),
           (dict(gate_kind=1), arg), (dict(gate=p), arg), (dict(scale=float("nan")), arg),
           (dict(eps=-1.0), arg), (dict(post_weight=None, pre_weight=None, u=None), arg),
           (dict(u=None), arg), (dict(pre_weight=None), arg), (dict(x=None), arg), (dict(f=None), arg),
           (dict(pre_rstd=None), arg), (dict(post_mean=None), arg), (dict(post_weight=None, post_bias=p), arg),
           (dict(x=p + 8), unsupported), (dict(u=p + 4), unsupported), (dict(pre_weight=p + 4), unsupported)]
    for kw, want in fwd:
        assert call("moe_block_norm_fwd", **kw) == want, kw
        assert B.moe_last_error()
    back = dict(du=p, dres=p, dx=p, df=p, d_post_weight=p, d_pre_weight=p, ws=p, ws_bytes=1 << 30)
    bwd = [(dict(du=None), arg), (dict(dx=None), arg), (dict(d_pre_weight=None), arg),
           (dict(d_post_weight=None), arg), (dict(ws_bytes=16), arg), (dict(ws=None), arg),
           (dict(gate_kind=1, gate=p), arg), (dict(ws=p + 8), unsupported), (dict(df=p + 2), unsupported),
           (dict(pre_weight=None, dres=None), arg)]
    for kw, want in bwd:
        assert call("moe_block_norm_bwd", **dict(back, **kw)) == want, kw
    assert L.moe_block_norm_fwd(None, None) == arg and L.moe_block_norm_bwd(None, None) == arg
    assert B.moe_block_norm_bwd_workspace_size(4, 60, B.MOE_F32) == 0
