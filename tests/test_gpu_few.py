"""The layer for a few tokens: its routing is moe_route_mask's bit for bit, its output that of
64-bit arithmetic on the same routes.

Tolerance, u = 2^-24, h half a step of the layer's type: a first projection's sum of d
products is off by at most d u times the sum of magnitudes (any order of summation), so
h = s silu(g) v is off by s (1.1 |v| dg + |silu(g)| dv) (|silu'| <= 1.1) and a few u and h of
itself; y sums |W_d| of that, H K' u of its own sum of magnitudes, and h of y.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.layer import (InferenceMoELayer, LayerNorm, ResidentMoELayer, mxfp4_dequantize,
                                        mxfp4_quantize)

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def case(T, d, E, E_r, k, H, Hs=0, dtype="bf16", mx=False, gate="softmax_topk", expert="swiglu",
         bias=False, tau=1.0):
    return dict(T=T, d=d, E=E, E_r=E_r, k=k, H=H, Hs=Hs, dtype=dtype, mx=mx, gate=gate, expert=expert,
                bias=bias, tau=tau)


CASES = [
    case(1, 64, 1, 1, 1, 64), case(1, 512, 16, 16, 4, 192, 128), case(2, 320, 8, 3, 2, 128, bias=True),
    case(15, 256, 64, 20, 6, 64, 64), case(16, 192, 65, 65, 8, 64, gate="softmax"),
    case(17, 128, 256, 100, 8, 128, gate="sigmoid", expert="silu"), case(32, 576, 12, 12, 3, 64, tau=0.5),
    case(33, 128, 32, 9, 4, 192, 320), case(48, 256, 40, 40, 6, 64, 64, expert="silu", bias=True),
    case(49, 64, 8, 1, 2, 128), case(64, 128, 130, 64, 8, 64, 64), case(5, 2048, 16, 5, 2, 704, 1408),
    case(9, 128, 8, 0, 2, 64, 64), case(9, 128, 8, 0, 2, 64),
    case(1, 64, 4, 4, 2, 64, dtype="f32"), case(7, 64, 8, 4, 2, 128, dtype="f32", bias=True),
    case(19, 264 + 56, 40, 17, 5, 64, 128, dtype="f32", expert="silu"),
    case(64, 192, 256, 256, 8, 64, dtype="f32", gate="softmax", tau=2.0),
    case(40, 128, 16, 7, 3, 64, 64, dtype="f32", gate="sigmoid"),
    case(1, 512, 16, 16, 4, 192, 128, mx=True), case(16, 192, 64, 30, 6, 64, 64, mx=True),
    case(30, 320, 24, 24, 3, 704, mx=True, expert="silu"), case(64, 128, 16, 10, 8, 128, 192, mx=True),
    case(47, 64, 8, 3, 2, 64, mx=True, gate="sigmoid", bias=True),
]


def make(c, seed=0):
    g = torch.Generator().manual_seed(seed + c["T"] + c["d"])
    dt, r1 = DT[c["dtype"]], 2 if c["expert"] == "swiglu" else 1
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dt).cuda()
    ids = torch.randperm(c["E"], generator=g)[: c["E_r"]]
    res = torch.zeros(c["E"], dtype=torch.uint8)
    res[ids] = 1
    t = dict(x=n(c["T"], c["d"]), w_router=n(c["E"], c["d"], std=0.1), res=res,
             bias=torch.randn(c["E"], generator=g).cuda() if c["bias"] else None)
    w = dict(w_gate_up=n(c["E_r"], r1 * c["H"], c["d"], std=0.1), w_down=n(c["E_r"], c["d"], c["H"], std=0.1))
    if c["Hs"]:
        w.update(shared_gate_up=n(1, r1 * c["Hs"], c["d"], std=0.1), shared_down=n(1, c["d"], c["Hs"], std=0.1))
    if c["mx"]:
        w = {name: mxfp4_quantize(v) for name, v in w.items()}
    t["w"] = w
    return t


def build(c, t):
    return InferenceMoELayer(c["k"], t["res"], t["w_router"], router_bias=t["bias"], gate=c["gate"],
                             inv_tau=1 / c["tau"], expert=c["expert"], **t["w"])


def routing(c, t, T):
    """moe_route_mask on the first T tokens."""
    f = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")
    i32 = torch.int32
    out = (f(T, c["E"]), f(T, c["k"], dt=i32), f(T, c["k"]), f(T, c["k"], dt=i32))
    B.moe_route_mask(t["x"], t["w_router"], t["bias"], B.dtype_code(t["x"]), T, c["d"], c["E"], c["k"],
                     1 / c["tau"], B.GATES[c["gate"]], t["res"].cuda(), *out)
    return out


def values(w):
    return (mxfp4_dequantize(*w, torch.float32) if isinstance(w, tuple) else w).double()


def reference(c, t, topk_w, local):
    """(y, its bound) in 64 bits on the given routes."""
    x, h_step = t["x"].double(), torch.finfo(DT[c["dtype"]]).eps / 2
    T, d, w = c["T"], c["d"], {k: values(v) for k, v in t["w"].items()}
    y = torch.zeros(T, d, dtype=torch.float64, device="cuda")
    err, mag = torch.zeros_like(y), torch.zeros_like(y)

    def block(xt, s, wgu, wd):
        H = wd.shape[1]
        a, da = xt @ wgu.T, d * U * (xt.abs() @ wgu.abs().T)
        g, dg = a[:, :H], da[:, :H]
        act = g / (1 + torch.exp(-g))
        if c["expert"] == "swiglu":
            v, dv = a[:, H:], da[:, H:]
            h, dh = act * v, 1.1 * dg * (v.abs() + dv) + act.abs() * dv
        else:
            h, dh = act, 1.1 * dg
        h, dh = s * h, s * dh
        dh = dh + (h_step + 16 * U) * (h.abs() + dh)
        return h @ wd.T, dh @ wd.abs().T, h.abs() @ wd.abs().T

    total = c["Hs"]
    for r in range(c["E_r"]):
        tok, j = (local == r).nonzero(as_tuple=True)
        if tok.numel():
            o = block(x[tok], topk_w[tok, j].double()[:, None], w["w_gate_up"][r], w["w_down"][r])
            for acc, v in zip((y, err, mag), o):
                acc.index_add_(0, tok, v)
    if c["Hs"]:
        for acc, v in zip((y, err, mag), block(x, 1.0, w["shared_gate_up"][0], w["shared_down"][0])):
            acc += v
    n = c["Hs"] + c["k"] * c["H"]
    return y, (err + n * U * (mag + err)) * (1 + h_step) + h_step * y.abs()


def check(c, t, L):
    y = L.few(t["x"])
    torch.cuda.synchronize()
    logits, idx, w, local = routing(c, t, c["T"])
    assert torch.equal(L.logits, logits) and torch.equal(L.topk_idx, idx)
    assert torch.equal(L.topk_w, w) and torch.equal(L.topk_local, local)
    ref, tol = reference(c, t, w, local)
    over = ((y.double() - ref).abs() - tol).max().item()
    assert torch.isfinite(y).all() and over <= 0, f"y: {over:.3e} past its bound"


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_few_matches_64_bits(gpu_lib, c):
    print("[few]", c, flush=True)
    t = make(c)
    check(c, t, build(c, t))


WIDE = [
    # d of 4096 and more: blocks of 16 columns of y; the router's other paths past 2048 and 4096
    case(1, 4096, 8, 4, 2, 64, 64), case(17, 4160, 8, 5, 2, 192, 64), case(33, 4096, 100, 12, 4, 64, expert="silu"),
    case(64, 4160, 6, 3, 3, 64, 128, bias=True), case(40, 8192, 33, 4, 2, 64), case(9, 2112, 48, 20, 4, 64, 64),
    case(50, 2112, 130, 20, 8, 64), case(5, 4160, 6, 3, 2, 64, 64, dtype="f32"),
    case(16, 4096, 8, 3, 2, 64, dtype="f32", expert="silu"), case(21, 4160, 8, 3, 2, 64, 64, dtype="f32"),
    case(60, 4096, 8, 3, 2, 64, dtype="f32"), case(3, 4096, 8, 4, 2, 192, 320, mx=True),
    case(8, 4160, 8, 4, 2, 320, mx=True), case(16, 4160, 8, 3, 2, 192, 64, mx=True, expert="silu"),
    case(17, 4096, 8, 3, 2, 64, 192, mx=True), case(40, 4160, 6, 3, 2, 192, 320, mx=True),
    case(64, 4096, 8, 5, 3, 64, mx=True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("c", WIDE, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_few_wide_rows(gpu_lib, c):
    test_few_matches_64_bits(gpu_lib, c)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_few_all_ghosts_and_one_expert_for_all(gpu_lib, mx):
    """Tokens that route to ghosts alone get exactly the shared output or 0; one expert may get
    every token."""
    for T, hot, E_r in ((20, [0, 1], 6), (64, [6, 7], 6), (64, [6, 3], 8)):
        c = case(T, 128, 8, E_r, 2, 64, mx=mx)
        t = make(c)
        t["res"] = torch.zeros(8, dtype=torch.uint8)
        t["res"][8 - E_r:] = 1
        t["bias"] = torch.zeros(8, device="cuda")
        t["bias"][hot] = 1e4
        c["bias"] = True
        L = build(c, t)
        check(c, t, L)
        if hot == [0, 1]:
            assert (L.topk_local == -1).all() and (L.y == 0).all()


@pytest.mark.gpu
def test_few_sizes_in_turn_bounds_and_repeats(gpu_lib):
    """One layer for changing numbers of tokens; nothing behind the last row of an output or of
    the workspace; the same bits whatever the workspace held."""
    c = case(64, 192, 24, 10, 4, 128, 64)
    t = make(c)
    L = build(c, t)
    whole = L.few(t["x"]).clone()
    for T in (0, 1, 16, 33, 64, 7):
        y = L.few(t["x"][:T])
        assert y.shape == (T, 192)
        # a token's output does not depend on the batch's size but for the order of the sums
        assert (y.double() - whole[:T].double()).abs().max().item() <= 0.02 * whole.abs().max().item() if T else True
        f = L._few
        pad = torch.full((T + 1, 192), 7.0, dtype=torch.bfloat16, device="cuda")
        idx = torch.full((T + 1, 4), -7, dtype=torch.int32, device="cuda")
        ws = torch.full((f.ws_bytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        keep = f.y, f.topk_idx, f.ws, f.logits, f.topk_w, f.topk_local
        f.y, f.topk_idx, f.ws, f.topk_w, f.topk_local = pad.data_ptr(), idx.data_ptr(), ws.data_ptr(), None, None
        B.moe_few_fwd(f)
        assert torch.equal(pad[:T], y) and (pad[T:] == 7).all() and (ws[f.ws_bytes:] == 0xFF).all()
        assert torch.equal(idx[:T], L.topk_idx) and (idx[T:] == -7).all()
        f.y, f.topk_idx, f.ws, f.logits, f.topk_w, f.topk_local = keep
        # without logits the workspace is larger
        f.logits = None
        n = B.moe_few_fwd_workspace_size(f)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        f.ws, f.y = ws.data_ptr(), pad.data_ptr()
        pad.fill_(7.0)
        bytes_before, f.ws_bytes = f.ws_bytes, n
        B.moe_few_fwd(f)
        assert torch.equal(pad[:T], y)
        f.ws_bytes = bytes_before
        f.y, f.topk_idx, f.ws, f.logits, f.topk_w, f.topk_local = keep


@pytest.mark.gpu
def test_few_more_residents_than_said(gpu_lib):
    """A resident set with more experts than E_r: the ones past it are ghosts, not reads past
    the weights."""
    c = case(30, 128, 16, 6, 4, 64)
    t = make(c)
    L = build(c, t)
    res = t["res"].clone()
    first = res.nonzero()[:, 0]
    res[15 if first[-1] != 15 else 14] = 1
    res = res.cuda()
    L._few.resident = res.data_ptr()
    L.few(t["x"])
    assert L.topk_local.max().item() < 6 and torch.isfinite(L.y).all()


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_few_graph_streams_and_two_at_once(gpu_lib, mx):
    """Captured and replayed with other tokens between eager calls; two layers on two streams."""
    c = case(12, 256, 16, 16, 4, 128, 64, mx=mx)
    a, b = make(c, 1), make(c, 2)
    La, Lb = build(c, a), build(c, b)
    xs = [torch.randn(12, 256, device="cuda").to(torch.bfloat16) for _ in range(4)]
    ref_a = [La.few(x).clone() for x in xs]
    ref_b = [Lb.few(x).clone() for x in xs]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for x, ra, rb in zip(xs, ref_a, ref_b):
            ya, yb = La.few(x, stream=s1), Lb.few(x, stream=s2)
            torch.cuda.synchronize()
            assert torch.equal(ya, ra) and torch.equal(yb, rb)
    live = xs[0].clone()
    La.few(live)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        La.few(live)
    for x, r in list(zip(xs, ref_a)) * 2:
        live.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(La.y, r)
        assert torch.equal(La.few(x), r)


@pytest.mark.gpu
def test_few_graph_outlives_other_sizes(gpu_lib):
    """A captured call of 5 tokens, replayed after eager calls of more and fewer and after other
    tensors were made and dropped."""
    c = case(5, 192, 16, 8, 2, 128, 64)
    L = build(c, make(c, 4))
    x = torch.randn(5, 192, device="cuda").to(torch.bfloat16)
    ref = L.few(x).clone()
    L.few(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = L.few(x)
    for T in (64, 1, 33, 5):
        more = torch.randn(T, 192, device="cuda").to(torch.bfloat16)
        more[:min(T, 5)] = x[:T]
        got = L.few(more)
        junk = [torch.full((1 << 18,), 3.0, device="cuda") for _ in range(8)]
        assert torch.isfinite(got).all() and L.topk_idx.shape == (T, 2)
        assert T != 5 or torch.equal(got, ref)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and all((j == 3.0).all() for j in junk)


@pytest.mark.gpu
def test_few_infinities_in_a_cut_step(gpu_lib):
    """MXFP4 widths that are no multiple of a step: an infinity is multiplied by its own weights
    alone.  Weights of ones (and gates of 1): the sums are infinite, no NaN; the other token
    stays as it is."""
    for d, H in ((64, 64), (320, 192), (448, 64)):
        q = lambda *s: mxfp4_quantize(torch.ones(*s, dtype=torch.bfloat16, device="cuda"))
        L = InferenceMoELayer(1, np.array([1]), torch.ones(1, d, dtype=torch.bfloat16, device="cuda"),
                              q(1, 2 * H, d), q(1, d, H), gate="sigmoid")
        x = torch.ones(2, d, dtype=torch.bfloat16, device="cuda")
        clean = L.few(x).clone()
        for at in range(0, d, 8):
            x[0] = 1.0
            x[0, at + at // 8 % 8] = float("inf")
            y = L.few(x)
            assert torch.equal(y[1], clean[1])
            assert L.topk_w[0].item() == 1 and (y[0] == float("inf")).all(), (d, H, at)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,mx", [("bf16", False), ("f32", False), ("bf16", True)])
def test_few_what_is_not_finite_stays_where_it_is(gpu_lib, dtype, mx):
    """NaN tokens: their rows alone, with moe_route_mask's routes; a NaN in an expert's weights:
    the tokens that are routed to it."""
    c = case(20, 192, 24, 10, 3, 128, 64, dtype=dtype, mx=mx)
    t = make(c, 6)
    L = build(c, t)
    clean = L.few(t["x"]).clone()
    x = t["x"]
    t["x"] = x.clone()
    t["x"][4], t["x"][11, 7], t["x"][19, 100] = float("nan"), float("nan"), float("-inf")
    y = L.few(t["x"])
    logits, idx, w, local = routing(c, t, 20)
    assert torch.equal(L.topk_idx, idx) and torch.equal(L.topk_local, local)
    for a, b in ((L.logits, logits), (L.topk_w, w)):
        assert torch.equal(a.nan_to_num(7.0, 8.0, 9.0), b.nan_to_num(7.0, 8.0, 9.0))
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[[4, 11, 19]] = True
    assert torch.equal(y[~bad], clean[~bad]) and not torch.isfinite(y[bad]).any()
    for name, at in (("w_gate_up", (6, 200, 70)), ("w_down", (2, 190, 127))):
        w = dict(t["w"])
        v = (mxfp4_dequantize(*w[name]) if mx else w[name]).clone()
        v[at] = float("nan")
        w[name] = mxfp4_quantize(v) if mx else v
        M = build(c, dict(t, w=w))
        y = M.few(x)
        hit = (M.topk_local == at[0]).any(1)
        assert hit.any() and not hit.all() and torch.equal(y[~hit], clean[~hit])
        # (a row of W_d: one column of y)
        assert y[hit][:, at[1] if name == "w_down" else slice(None)].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_agrees_with_the_training_layer(gpu_lib, dtype):
    """Behind the pre-norm, on the same weights: the training layer's forward, whose routes it
    takes bit for bit.  That layer also rounds each route's output and the sum (two more
    half steps, on at most k + 1 terms)."""
    c = case(37, 256, 24, 10, 4, 128, 64, dtype=dtype)
    t = make(c)
    N = LayerNorm(37, 256, dtype=DT[dtype], bias=False)
    t["x"] = N.forward(t["x"], torch.ones(256, device="cuda")).clone()
    L = build(c, t)
    R = ResidentMoELayer(37, 256, 24, 4, 128, t["res"], dtype=DT[dtype], n_shared_hidden=64)
    y = R.forward(t["x"], t["w_router"], **t["w"])
    check(c, t, L)
    assert torch.equal(L.topk_idx, R.topk_idx) and torch.equal(L.topk_w, R.topk_w)
    ref, tol = reference(c, t, R.topk_w, R.topk_local)
    h = torch.finfo(DT[dtype]).eps / 2
    # its route outputs are below mag in sum; bounded here by the largest of |y| and tol's scale
    scale = ref.abs().amax(dim=1, keepdim=True) * (c["k"] + 1)
    assert ((L.y.double() - y.double()).abs() <= 2 * tol + 2 * h * scale).all()


def kernel_us(L, x, name, n=10):
    """The least of n times of one kernel of a call, us."""
    L.few(x)
    torch.cuda.synchronize()
    best = float("inf")
    for _ in range(n):
        B.moe_timing_enable(8)
        try:
            L.few(x)
            torch.cuda.synchronize()
            best = min(best, B.moe_timing_collect()[name][1] * 1e3)
        finally:
            B.moe_timing_enable(0)
    return best


def shared_only(dtype="bf16", mx=False, d=1024, Hs=1 << 16):
    """A layer of shared experts alone, so large (100 MB in 4 bits) that reading them
    is all of its time."""
    dt = DT[dtype]
    q = mxfp4_quantize if mx else lambda w: w
    w = lambda *s: q(torch.full(s, 0.5, dtype=dt, device="cuda"))
    none = lambda *s: q(torch.empty(0, *s, dtype=dt, device="cuda"))
    return InferenceMoELayer(1, np.array([0]), torch.ones(1, d, dtype=dt, device="cuda"), none(128, d), none(d, 64),
                             shared_gate_up=w(1, 2 * Hs, d), shared_down=w(1, d, Hs))


@pytest.mark.gpu
def test_few_shared_items_once(gpu_lib):
    """Four tokens' shared first projections from MXFP4 are made once: 16 tokens read the weights
    twice, four of them once, in little more than half of the time (made twice, in all of it)."""
    L = shared_only(mx=True)
    x = torch.ones(16, 1024, dtype=torch.bfloat16, device="cuda")
    few, more = kernel_us(L, x[:4], "few_gu"), kernel_us(L, x, "few_gu")
    print(f"[few] 4 tokens {few:.1f} us, 16 {more:.1f}", flush=True)
    assert few < 0.8 * more


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,mx,T,more,passes,many", [("bf16", True, 8, 16, 1, 2), ("bf16", True, 24, 64, 3, 8),
                                                         ("f32", False, 24, 64, 1, 2)])
def test_few_passes_by_tokens(gpu_lib, dtype, mx, T, more, passes, many):
    """Shared weights are read as often as the tokens need: T tokens' passes over them against
    more tokens' (all readings made by both, whatever T, the times were the same).  The bound
    lies halfway between the passes' ratio and one."""
    L = shared_only(dtype, mx)
    x = torch.ones(more, 1024, dtype=DT[dtype], device="cuda")
    for name in ("few_gu", "few_down"):
        few, all_ = kernel_us(L, x[:T], name), kernel_us(L, x, name)
        print(f"[few] {name} {T} tokens {few:.1f} us, {more} {all_:.1f}", flush=True)
        assert few < (1 + passes / many) / 2 * all_, name


def _few(**kw):
    p = 256  # a fake, never dereferenced address
    a = dict(dtype=B.MOE_BF16, weights=0, activation=0, gate=0, T=4, d=128, E=8, k=2, E_r=4, H=64, Hs=64,
             inv_tau=1.0, x=p, w_router=p, resident=p, w_gate_up=p, w_down=p, shared_gate_up=p,
             shared_down=p, y=p, ws=p)
    a.update(kw)
    f = B.moe_few(**a)
    if "ws_bytes" not in kw:
        f.ws_bytes = B.moe_few_fwd_workspace_size(f)
    return f


def test_few_refusals():
    if torch.cuda.device_count() > 0:
        pytest.skip("host-only rejection test: runs where no GPU is visible")
    fwd = lambda **kw: B.lib().moe_few_fwd(C.byref(_few(**kw)), None)
    assert B.lib().moe_few_fwd(None, None) == -1 and B.lib().moe_few_fwd_workspace_size(None) == 0
    for kw in (dict(dtype=4), dict(T=65), dict(k=9, E=16), dict(d=96), dict(H=32), dict(Hs=96),
               dict(weights=1, dtype=B.MOE_F32), dict(d=1 << 16, H=1 << 16),
               dict(d=64, H=1 << 21, T=64, k=8, E=16), dict(x=260), dict(w_down=264), dict(ws=128)):
        assert fwd(**kw) == -2, kw
    for kw in (dict(T=-1), dict(E=0), dict(E=257), dict(k=0), dict(k=9), dict(E_r=9), dict(gate=3),
               dict(activation=2), dict(weights=2), dict(inv_tau=0.0), dict(inv_tau=float("inf")),
               dict(x=None), dict(y=None), dict(w_router=None), dict(resident=None), dict(w_down=None),
               dict(shared_down=None), dict(weights=1), dict(ws=None), dict(ws_bytes=10), dict(Hs=-64)):
        assert fwd(**kw) == -1, kw
    sizes = [B.moe_few_fwd_workspace_size(_few(T=T)) for T in (0, 1, 16, 64)]
    assert sizes == sorted(sizes) and B.moe_few_fwd_workspace_size(_few(T=65)) == 0
    assert B.moe_few_fwd_workspace_size(_few(logits=256)) < B.moe_few_fwd_workspace_size(_few())


def test_inference_layer_workspace_of_wide_experts():
    """Experts so wide that 64 tokens of 8 routes are past the library's limit: fewer are taken,
    and the workspace is theirs."""
    H = 1 << 20
    L = InferenceMoELayer(8, np.zeros(8), torch.zeros(8, 64), torch.zeros(0, 2 * H, 64), torch.zeros(0, 64, H))
    L._size(1)
    need = [B.moe_few_fwd_workspace_size(L._few)]
    L._size(63)
    need.append(B.moe_few_fwd_workspace_size(L._few))
    assert 0 < need[0] < need[1] == L._few.ws_bytes == L._ws.numel()
    L._size(64)
    assert B.moe_few_fwd_workspace_size(L._few) == 0 and "2^29" in B.moe_last_error()


def test_inference_layer_checks():
    """Wrong shapes, types and mixtures are refused when the layer is built (on any device)."""
    E, d, H = 6, 128, 64
    w = dict(w_gate_up=torch.zeros(3, 2 * H, d), w_down=torch.zeros(3, d, H))
    res, wr = np.array([1, 0, 1, 0, 1, 0]), torch.zeros(E, d)
    InferenceMoELayer(2, res, wr, **w)
    bad = [dict(w, w_down=torch.zeros(3, H, d)), dict(w, w_gate_up=w["w_gate_up"].bfloat16()),
           dict(w, w_gate_up=w["w_gate_up"][:2]), dict(w, shared_down=torch.zeros(1, d, H)),
           dict(w, w_down=(torch.zeros(3, d, H // 2, dtype=torch.uint8), torch.zeros(3, d, 4, dtype=torch.uint8))),
           dict(w, router_bias=torch.zeros(E, dtype=torch.bfloat16)), dict(w, expert="silu")]
    for kw in bad:
        with pytest.raises(ValueError):
            InferenceMoELayer(2, res, wr, **kw)
    with pytest.raises(ValueError):
        InferenceMoELayer(2, res[:5], wr, **w)
    with pytest.raises(ValueError):
        InferenceMoELayer(2, res, wr, **w).few(torch.zeros(4, d))  # not on a GPU
