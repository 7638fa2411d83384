"""The expert FFN in MXFP4 against 64-bit arithmetic on the same codes.

Tolerance, u = 2^-24: a first projection's sum of d products is off by at most d u times the
sum of magnitudes (any order of summation), which moves h by dh = 1.1 |U| dG + |silu(G)| dU
(|silu'| <= 1.1); silu itself is off by a few u (exp2 and the reciprocal are good to 2 u, and
three roundings) and, from the rounding of G log2 e, by 1.45 |G| u of itself.  h becomes codes: where its border or its block's
scale lies within dh the neighbouring code is as right, so each quantised h lies between the
least and the greatest of its four candidates (h -+ dh under the scales of the block's
largest value -+ its dh).  y sums |W_d| of that range, H u of its own sum of magnitudes and
half a bf16 step."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2606_19025_amd import binding as B
from paper_2606_19025_amd.layer import MxFFN, ResidentMoELayer, mxfp4_dequantize, mxfp4_quantize

U, HALF = 2.0 ** -24, 2.0 ** -8
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def to_grid(v, s):
    """v [rows, blocks, 32] rounded to codes under scale exponents s [rows, blocks, 1]."""
    a = v * pow2(-s)
    d = (a.abs()[..., None] - GRID.to(v.device)).abs()
    d[..., 1::2] += 1e-12  # ties to the even code
    return GRID.to(v.device)[d.argmin(dim=-1)] * torch.sign(a) * pow2(s)


def quantised(h, dh):
    """(value, least, greatest) of h's codes where h is known to dh."""
    b, db = h.reshape(len(h), -1, 32), dh.reshape(len(h), -1, 32)
    top = lambda t: (torch.frexp(t.amax(dim=2, keepdim=True).clamp(min=2.0 ** -126)).exponent - 3).clamp(min=-127)
    mid = to_grid(b, top(b.abs()))
    c = [to_grid(b + s * db, e) for s in (-1, 1)
         for e in (top((b.abs() - db).clamp(min=0)), top(b.abs() + db))]
    c = torch.stack(c + [mid])
    return tuple(v.reshape(h.shape) for v in (mid, c.amin(0), c.amax(0)))


def make(sizes, d, H, expert="swiglu", seed=0, extra=0):
    g = torch.Generator().manual_seed(seed + d + H + sum(sizes))
    r1, ng = 2 if expert == "swiglu" else 1, len(sizes)
    n = lambda *s, std=1.0: torch.randn(*s, generator=g).mul(std).cuda()
    cap = sum(sizes) + extra
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32).cuda()
    return (n(cap, d).bfloat16(), off, mxfp4_quantize(n(ng, r1 * H, d, std=0.1)),
            mxfp4_quantize(n(ng, d, H, std=0.1)))


def reference(x, sizes, gu, dn, expert):
    xq = mxfp4_dequantize(*mxfp4_quantize(x), torch.float32).double()
    wgu, wd = (mxfp4_dequantize(*w, torch.float32).double() for w in (gu, dn))
    y, tol, at = torch.zeros(len(x), wd.shape[1], dtype=torch.float64, device="cuda"), None, 0
    tol = torch.zeros_like(y)
    for g, n in enumerate(sizes):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        xr, w, d2 = xq[rows], wgu[g], wd[g]
        H = d2.shape[1]
        a, da = xr @ w.T, xr.shape[1] * U * (xr.abs() @ w.abs().T)
        G, dG = a[:, :H], da[:, :H]
        act = G / (1 + torch.exp(-G))
        if expert == "swiglu":
            h, dh = act * a[:, H:], 1.1 * dG * (a[:, H:].abs() + da[:, H:]) + act.abs() * da[:, H:]
        else:
            h, dh = act, 1.1 * dG
        mid, lo, hi = quantised(h, dh + (16 + 1.5 * G.abs()) * U * (h.abs() + dh))
        y[rows] = mid @ d2.T
        tol[rows] = (torch.maximum(hi - mid, mid - lo) + H * U * mid.abs()) @ d2.abs().T
    return y, (tol * (1 + HALF) + HALF * y.abs())


SIZES = [([1], 64, 64, "swiglu"), ([5, 0, 3], 128, 192, "swiglu"), ([64, 65, 63, 1, 0], 320, 64, "silu"),
         ([300], 576, 704, "swiglu"), ([0, 0, 7], 64, 320, "silu"), ([130, 1, 257, 40], 192, 128, "swiglu"),
         ([256] * 3 + [300, 511], 256, 1344, "swiglu"), ([2000, 1, 700], 448, 640, "silu"),
         ([3] * 40, 192, 192, "swiglu")]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,d,H,expert", SIZES)
def test_mxffn_matches_64_bits(gpu_lib, sizes, d, H, expert):
    print("[mxffn]", sizes[:8], d, H, expert, flush=True)
    x, off, gu, dn = make(sizes, d, H, expert, extra=3)
    n = sum(sizes)
    L = MxFFN(n + 3, gu, dn, expert=expert)
    L.y.fill_(7.0)
    L.ws.fill_(0xFF)
    L.xq.fill_(0xA5)
    L.xs.fill_(0xFF)
    y = L.forward(x, off)
    ref, tol = reference(x[:n], sizes, gu, dn, expert)
    assert torch.isfinite(y).all()
    over = ((y[:n].double() - ref).abs() - tol).max().item()
    assert over <= 0, f"{over:.3e} past its bound"
    assert (y[n:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d,H,expert", [(2112, 576, "swiglu"), (2048, 1088, "silu"), (512, 64, "swiglu"),
                                        (4160, 512, "silu"), (2304, 1216, "swiglu")])
def test_mxffn_large_tiles(gpu_lib, d, H, expert):
    """Room for so many rows that the large tiles are taken, and few of them there (the others
    NaN): ragged groups, cut and whole last steps of the reduction, one step and many."""
    sizes = [300, 0, 401, 1, 257]
    print("[mxffn]", sizes, d, H, expert, flush=True)
    x, off, gu, dn = make(sizes, d, H, expert)
    n, cap = sum(sizes), 33000
    L = MxFFN(cap, gu, dn, expert=expert)
    L.y.fill_(7.0)
    L.ws.fill_(0xFF)
    room = torch.full((cap, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    room[:n] = x
    y = L.forward(room, off)
    ref, tol = reference(x, sizes, gu, dn, expert)
    assert torch.isfinite(y[:n]).all()
    over = ((y[:n].double() - ref).abs() - tol).max().item()
    assert over <= 0, f"{over:.3e} past its bound"
    assert (y[n:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,d,H,expert", [([1] * 256, 192, 704, "swiglu"), ([0, 1] * 64, 1088, 320, "silu"),
                                              ([127] * 48, 576, 1408, "swiglu"), ([129] * 48, 576, 1408, "swiglu")])
def test_mxffn_few_rows_in_many_groups(gpu_lib, sizes, d, H, expert):
    """Groups of one row and fewer, and of half a large tile and one more (the border of the tiles'
    choice)."""
    test_mxffn_matches_64_bits(gpu_lib, sizes, d, H, expert)


def tiles(sizes, bm, N, bn):
    return sum(-(-n // bm) for n in sizes) * -(-N // bn)


@pytest.mark.gpu
@pytest.mark.parametrize("expert,H", [("swiglu", 1088), ("silu", 2112)])
@pytest.mark.parametrize("large", [True, False])
def test_mxffn_blocks_take_several_tiles(gpu_lib, large, expert, H):
    """More tiles than blocks (256 of large ones, 512 of small ones) in both projections: a block
    loads its next tile while it stores one."""
    d = 1216 if large else 1600
    if not large:
        H = 832 if expert == "swiglu" else 1664
    sizes = [2300, 0, 1, 4097, 255, 5000, 513, 7000] if large else [65 + 7 * i % 60 for i in range(40)]
    N = 2 * H if expert == "swiglu" else H
    for cols in (N, d):
        # the large tiles are taken from one per CU on
        if large:
            assert tiles(sizes, 256, cols, 256) > 256 and sum(sizes) // 256 * -(-cols // 256) > 256
        else:
            assert tiles(sizes, 64, cols, 128) > 512 and (sum(sizes) // 256 + 20) * -(-cols // 256) < 256
    print("[mxffn]", len(sizes), sum(sizes), d, H, expert, flush=True)
    x, off, gu, dn = make(sizes, d, H, expert, extra=5)
    n = sum(sizes)
    L = MxFFN(n + 5, gu, dn, expert=expert)
    L.y.fill_(7.0)
    L.ws.fill_(0xFF)
    y = L.forward(x, off).clone()
    ref, tol = reference(x[:n], sizes, gu, dn, expert)
    assert torch.isfinite(y).all()
    over = ((y[:n].double() - ref).abs() - tol).max().item()
    assert over <= 0, f"{over:.3e} past its bound"
    assert (y[n:] == 7).all() and torch.equal(L.forward(x, off), y)


@pytest.mark.gpu
def test_mxffn_offsets_out_of_range_and_empty(gpu_lib):
    """Groups are clamped to [0, cap]; no groups or no rows write nothing."""
    x, off, gu, dn = make([20, 30, 14], 128, 64)
    L = MxFFN(64, gu, dn)
    whole = L.forward(x, off).clone()
    L.y.fill_(7.0)
    L.forward(x, torch.tensor([-5, 20, 50, 900], dtype=torch.int32, device="cuda"))
    assert torch.equal(L.y, whole)
    L.y.fill_(7.0)
    L.forward(x, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert (L.y == 7).all()
    L.forward(x, torch.tensor([10, 10, 40, 40], dtype=torch.int32, device="cuda"))
    assert (L.y[:10] == 7).all() and (L.y[40:] == 7).all() and torch.equal(L.y[20:40], whole[20:40])
    E = MxFFN(0, gu, dn)
    assert E.forward(x[:0], off).shape == (0, 128)


@pytest.mark.gpu
def test_mxffn_and_few_refuse_what_is_no_tensor_of_rows(gpu_lib):
    """Before anything is launched, and without a trace in the layer's outputs."""
    from paper_2606_19025_amd.layer import InferenceMoELayer
    x, off, gu, dn = make([20, 30, 14], 128, 64)
    F = MxFFN(64, gu, dn)
    whole = F.forward(x, off)
    for bad in (None, 3, x.half(), x.double(), x[:63], x[:, :64], x.T.contiguous().T, x.cpu()):
        with pytest.raises(ValueError):
            F.forward(bad, off)
    for bad in (None, off.long(), off[:3], off.cpu()):
        with pytest.raises(ValueError):
            F.forward(x, bad)
    L = InferenceMoELayer(2, np.ones(3), torch.ones(3, 128, dtype=torch.bfloat16, device="cuda"), gu, dn)
    y = L.few(x).clone()
    for bad in (None, 3, x[0], x[None], x.half(), x[:, :64], x.float(), torch.cat([x, x])):
        with pytest.raises(ValueError):
            L.few(bad)
    assert torch.equal(L.few(x), y) and torch.equal(F.forward(x, off), whole)


@pytest.mark.gpu
def test_mxffn_nan_stays_in_its_rows(gpu_lib):
    x, off, gu, dn = make([100, 28], 128, 128)
    L = MxFFN(128, gu, dn)
    clean = L.forward(x, off).clone()
    x[17, 5], x[120, 100] = float("nan"), float("inf")
    y = L.forward(x, off)
    bad = torch.zeros(128, dtype=torch.bool, device="cuda")
    bad[[17, 120]] = True
    assert y[bad].isnan().all() and torch.equal(y[~bad], clean[~bad])


@pytest.mark.gpu
def test_mxffn_silu_at_its_lower_end(gpu_lib):
    """Gate sums of -82 to -96 under up projections of 2^107: past -87.3 the exponential or its
    reciprocal leaves fp32's normal numbers, and silu, at most 1.03e-36 there, may be 0 or off by
    that much, which is added to the header's bound.  Every product and sum is exact (x of ones,
    the gate's weights -0.5 and -0.75), W_d the identity: y is h's codes, exact in bf16."""
    d = H = 128
    wg = torch.full((H, d), -0.5, device="cuda")
    for j in range(H):
        wg[j, : 72 + 56 * j // H] = -0.75
    wu = torch.full((H, d), 2.0 ** 100, device="cuda")
    gu, dn = mxfp4_quantize(torch.cat([wg, wu])[None]), mxfp4_quantize(torch.eye(d, device="cuda")[None])
    y = MxFFN(3, gu, dn).forward(torch.ones(3, d, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda"))
    g = wg.double().sum(1)[None]
    u = 2.0 ** 107
    h = g / (1 + torch.exp(-g)) * u
    mid, lo, hi = quantised(h, (16 + 1.5 * g.abs()) * U * h.abs() + 1.1e-36 * u)
    assert g.min() == -96 + 0.25 and g.max() == -82 and (mid[g < -89] != 0).any()
    assert ((y.double() >= lo) & (y.double() <= hi)).all()


@pytest.mark.gpu
def test_mxffn_graph_and_stream(gpu_lib):
    x, off, gu, dn = make([70, 0, 300], 256, 192)
    L = MxFFN(370, gu, dn)
    xs = [torch.randn(370, 256, device="cuda").bfloat16() for _ in range(3)]
    ref = [L.forward(v, off).clone() for v in xs]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for v, r in zip(xs, ref):
        y = L.forward(v, off, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(y, r)
    live = xs[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.forward(live, off)
    for v, r in list(zip(xs, ref)) * 2:
        live.copy_(v)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.y, r)
        assert torch.equal(L.forward(v, off), r)


@pytest.mark.gpu
@pytest.mark.parametrize("expert", ["swiglu", "silu"])
def test_mxffn_in_the_layers_chain(gpu_lib, expert):
    """Routed and dispatched by the training layer, the FFN from 4-bit experts, combined: the
    groups' offsets and the rows past the last one come from the device."""
    from .parity_helpers import dev
    from .test_gpu_parity import synth_inputs
    T, d, E, k, H = 333, 128, 12, 3, 128
    inp = synth_inputs(T, d, E, k, H, [0, 3, 5, 8], "bf16", seed=9)
    r1 = 2 if expert == "swiglu" else 1
    w = {n: dev(inp[n], torch.bfloat16) for n in ("w_router", "w_gate_up", "w_down")}
    w["w_gate_up"] = w["w_gate_up"][:, : r1 * H].contiguous()
    L = ResidentMoELayer(T, d, E, k, H, inp["resident"], expert=expert, canary=True)
    L.forward(dev(inp["x"], torch.bfloat16), **w)
    gu, dn = mxfp4_quantize(w["w_gate_up"]), mxfp4_quantize(w["w_down"])
    F = MxFFN(L.cap, gu, dn, expert=expert)
    F.y.fill_(float("nan"))
    F.forward(L.xp, L.offsets)
    y = torch.full((T, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.moe_combine_fwd(F.y, B.MOE_BF16, T, d, k, L.cap, L.topk_w, L.inv_perm, None, y)
    sizes, n = L.counts.tolist(), int(L.offsets[-1])
    ref, tol = reference(L.xp[:n], sizes, gu, dn, expert)
    assert ((F.y[:n].double() - ref).abs() <= tol).all() and F.y[n:].isnan().all()
    # combined: the same sum over the routes, rounded once more
    at = L.inv_perm.long()
    wt = torch.where(at >= 0, L.topk_w.double(), 0.0)[..., None]
    want, slack = ((wt * v[at.clamp(min=0)]).sum(1) for v in (ref, tol))
    assert ((y.double() - want).abs() <= slack * (1 + HALF) + HALF * want.abs() + 8 * U * want.abs() + 1e-30).all()


def test_mxffn_refusals():
    if torch.cuda.device_count() > 0:
        pytest.skip("host-only rejection test: runs where no GPU is visible")
    p = 256  # a fake, never dereferenced address
    need = B.moe_mxfp4_ffn_fwd_workspace_size(100, 128)
    assert need >= 100 * 64 + 100 * 4 and B.moe_mxfp4_ffn_fwd_workspace_size(-1, 128) == 0

    def f(**kw):
        a = dict(cap=100, d=128, H=128, n_groups=3, activation=0, x=p, x_scales=p, w_gate_up=p,
                 w_gate_up_scales=p, w_down=p, w_down_scales=p, offsets=p, y=p, ws=p, ws_bytes=need)
        a.update(kw)
        return B.lib().moe_mxfp4_ffn_fwd(C.byref(B.moe_mxfp4_ffn(**a)), None)

    assert B.lib().moe_mxfp4_ffn_fwd(None, None) == -1
    for kw in (dict(d=96), dict(H=32), dict(n_groups=257), dict(cap=1 << 22, d=4096), dict(x=p + 8),
               dict(y=p + 4), dict(x_scales=p + 2), dict(w_down_scales=p + 1), dict(ws=p + 16),
               dict(n_groups=256, H=8192, d=4096), dict(cap=1, n_groups=16, H=1 << 30, d=1 << 30)):
        kw = dict(kw, ws_bytes=1 << 40)
        assert f(**kw) == -2, kw
    for kw in (dict(cap=-1), dict(n_groups=-1), dict(d=0), dict(H=0), dict(activation=2), dict(offsets=None),
               dict(x=None), dict(x_scales=None), dict(y=None), dict(w_gate_up_scales=None), dict(w_down=None),
               dict(ws=None), dict(ws_bytes=need - 1)):
        assert f(**kw) == -1, kw


def test_mxffn_class_checks():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    gu, dn = (u8(2, 256, 64), u8(2, 256, 4)), (u8(2, 128, 64), u8(2, 128, 4))
    MxFFN(8, gu, dn)
    for a, b, kw in (((gu[0][:1], gu[1]), dn, {}), (gu, (dn[0], dn[1][:, :, :2]), {}), (gu, dn, dict(expert="silu")),
                     ((gu[0].float(), gu[1]), dn, {})):
        with pytest.raises(ValueError):
            MxFFN(8, a, b, **kw)
