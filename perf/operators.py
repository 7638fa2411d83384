"""Performance cases of the operators around the resident-expert MoE layer.

Each case is one pass through an operator, as a training or evaluation loop
calls it:

  norm    the layer's pre-norm (layer norm): forward, backward or both
  few     the whole MoE layer for a few tokens, from weights of the layer's own
          type or from MXFP4 ones
  quant   to MXFP4 (microscaled 4-bit floats) and back
  mxffn   the grouped expert FFN in MXFP4 of rows dispatched by expert, their
          quantisation included

With ``own`` false ``run`` computes the operators in elementary torch
operations, in 32 bits (router logits, whose order decides, in 64); with ``own``
true it calls the framework.  ``exact`` computes them in 64 bits from their
definitions.  Activations and upstream gradients are ~ N(0, 1), weights
~ N(0, 0.02), as in ``paper_2606_19025_amd.inputs``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5


def _norm(name, way, T, d, dtype="bf16", bias=True, res=True):
    return dict(name=name, family="norm", way=way, T=T, d=d, dtype=dtype, bias=bias, res=res)


def _few(name, T, d, E, E_r, k, H, Hs=0, dtype="bf16", weights="plain", gate="softmax_topk",
         expert="swiglu", bias=False):
    return dict(name=name, family="few", T=T, d=d, E=E, E_r=E_r, k=k, H=H, Hs=Hs, dtype=dtype,
                weights=weights, gate=gate, expert=expert, bias=bias)


def _quant(name, rows, cols, dtype="bf16"):
    return dict(name=name, family="quant", rows=rows, cols=cols, dtype=dtype)


def _mxffn(name, n, d, E_r, H, expert="swiglu", skew=False):
    return dict(name=name, family="mxffn", n=n, d=d, E_r=E_r, H=H, expert=expert, skew=skew)


def listed():
    return [
        # the pre-norm of one generated token: latency alone
        _norm("norm-fwd-one-bf16", "fwd", 1, 2048),
        # the pre-norm of the fine-grained workload's training step
        _norm("norm-step-fine-bf16", "both", 8192, 2048),
        # an fp32 run on a last, ragged micro-batch of an odd width, no bias
        _norm("norm-step-odd-f32", "both", 3001, 520, dtype="f32", bias=False),
        # the large workload's backward, with the residual stream's gradient
        _norm("norm-bwd-large-bf16", "bwd", 16384, 4096),
        # generation of one token with every expert of the fine-grained layer at
        # hand: six routed experts and the shared ones
        _few("few-one-bf16", 1, 2048, 64, 64, 6, 1408, Hs=2816),
        # evaluation of the fine-grained layer's worker on a handful of tokens
        _few("few-eval-bf16", 48, 2048, 64, 16, 6, 1408, Hs=2816),
        # the tiny fp32 layer: launches and latency
        _few("few-tiny-f32", 7, 64, 8, 4, 2, 128, dtype="f32"),
        # a batch of sequences generated together from 4-bit experts
        _few("few-batch-mxfp4", 16, 2048, 64, 32, 6, 1408, Hs=2816, weights="mxfp4"),
        # a worker's expert weights of the fine-grained workload to 4 bits
        _quant("quant-experts-bf16", 16 * 2816, 2048),
        # ragged fp32 rows of an odd width (704: 22 blocks)
        _quant("quant-odd-f32", 1531, 704, dtype="f32"),
        # the experts of the large workload (validation from 4-bit experts)
        _mxffn("mxffn-large", 65536, 4096, 32, 2048),
        # odd, unevenly loaded groups of the paper's own SiLU experts
        _mxffn("mxffn-odd-silu", 1531, 1024, 6, 704, expert="silu", skew=True),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of step between lo and hi, uniform over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    family = rng.choice(["norm", "norm", "few", "few", "few", "quant", "mxffn", "mxffn"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if family == "norm":
        T, d = _log(rng, 1, 16384), _log(rng, 64, 8192, 8)
        T = max(1, min(T, (1 << 26) // d))
        c = _norm("", rng.choice(["fwd", "bwd", "both"]), T, d, dtype, rng.random() < 0.7,
                  rng.random() < 0.5)
    elif family == "few":
        E = rng.choice([8, 16, 32, 48, 64, 128, 256])
        d, H = _log(rng, 64, 4096, 64), _log(rng, 64, 2816, 64)
        # the experts at hand hold at most 6e8 parameters
        E_r = max(1, min(int(E * rng.uniform(0.2, 1.0)), int(6e8 / (3 * d * H))))
        weights = "mxfp4" if dtype == "bf16" and rng.random() < 0.4 else "plain"
        c = _few("", _log(rng, 1, 64), d, E, E_r, rng.randint(1, min(8, E // 2)), H,
                 rng.choice([0, 0, H, 2 * H]), dtype, weights,
                 rng.choice(["softmax_topk", "softmax_topk", "softmax", "sigmoid"]),
                 rng.choice(["swiglu", "swiglu", "silu"]), rng.random() < 0.3)
    elif family == "quant":
        cols = _log(rng, 32, 8192, 32)
        c = _quant("", max(1, min(_log(rng, 1, 1 << 18), 9 * 10 ** 7 // cols)), cols, dtype)
    else:
        d, H = _log(rng, 64, 4096, 64), _log(rng, 64, 2816, 64)
        E_r = rng.choice([1, 2, 3, 6, 8, 12, 16, 32, 40])
        # at most a third of the largest listed case's operations
        n = max(8, min(_log(rng, 8, 65536), int(1.1e12 / (6 * d * H))))
        c = _mxffn("", n, d, E_r, H, rng.choice(["swiglu", "swiglu", "silu"]), rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------ MXFP4, plain
# E2M1 values by code (sign in bit 3); code 2i is the low nibble of byte i
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_stride(cols):
    """Bytes of a row of scales: whole words of four."""
    return (cols + 127) // 128 * 4


def _mx_blocks(x):
    """(signed E2M1 values [rows, cols / 32, 32], E8M0 codes [rows, cols / 32]) of x, in 32 bits.

    The scale is 2^(floor(log2 max) - 2), with the exponent read from the bits of the
    largest magnitude; scaling by it is exact, and a value becomes the nearest of the
    eight magnitudes (ties to the even code): the number of borders it has passed."""
    b = x.float().reshape(x.shape[0], -1, 32)
    top = b.abs().amax(dim=2).contiguous()
    s = ((top.view(torch.int32) >> 23) - 2).clamp_(min=0)
    v = b * ((254 - s) << 23).view(torch.float32).unsqueeze(2)
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0))
    code += (v < 0).to(torch.uint8) * 8
    return code, s.to(torch.uint8)


def _mx_values(code, s):
    """The 32-bit values of E2M1 codes [rows, blocks, 32] under E8M0 codes [rows, blocks]."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    s = s.int()
    scale = torch.where(s > 0, s << 23, 1 << 22).view(torch.float32)  # 2^(s - 127), s = 0 subnormal
    return (table[code.int()] * scale.unsqueeze(2)).flatten(1)


def _mx_pack(x):
    """(packed codes, scales) of x in the framework's layout."""
    code, s = _mx_blocks(x)
    code = code.flatten(1)
    scales = torch.zeros(x.shape[0], _mx_stride(x.shape[1]), dtype=torch.uint8, device=x.device)
    scales[:, : s.shape[1]] = s
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scales


def _mx_unpack(codes, scales):
    rows, cols = codes.shape[0], codes.shape[1] * 2
    code = torch.stack([codes & 15, codes >> 4], dim=2).reshape(rows, cols // 32, 32)
    return _mx_values(code, scales[:, : cols // 32])


# ------------------------------------------------------------------ inputs
class _Draw:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))
        self.r = np.random.default_rng(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        out = torch.empty(*shape, dtype=dtype, device="cuda")
        return out.normal_(mean, std, generator=self.g)

    def mx(self, n, rows, cols, std=0.02):
        """n matrices of weights in MXFP4: (codes [n, rows, cols / 2], scales [n, rows, stride])."""
        codes = torch.empty(n, rows, cols // 2, dtype=torch.uint8, device="cuda")
        scales = torch.empty(n, rows, _mx_stride(cols), dtype=torch.uint8, device="cuda")
        for i in range(n):
            codes[i], scales[i] = _mx_pack(self.normal(rows, cols, std=std))
        return codes, scales


def _projections(c):
    """Rows of the first projection, in units of H."""
    return 1 if c["expert"] == "silu" else 2


def prepare(case, seed):
    c, D = case, _Draw(seed)
    dt = DTYPES[c.get("dtype", "bf16")]
    if c["family"] == "norm":
        T, d = c["T"], c["d"]
        # activations of a residual stream: a row mean of its own, features of uneven scale
        x = (D.normal(T, d) * D.normal(d, std=0.3).exp_() + D.normal(T, 1, std=0.5)).to(dt)
        s = dict(case=c, x=x, w=D.normal(d, std=0.1, mean=1.0),
                 b=D.normal(d, std=0.1) if c["bias"] else None)
        if c["way"] != "fwd":
            s["dy"] = D.normal(T, d, dtype=dt)
            s["dres"] = D.normal(T, d, dtype=dt) if c["res"] else None
        if c["way"] == "bwd":  # what the forward left
            xd = x.double()
            mean = xd.mean(dim=1)
            s["mean"] = mean.float()
            s["rstd"] = (((xd - mean[:, None]) ** 2).mean(dim=1) + EPS).rsqrt().float()
        return s
    if c["family"] == "few":
        d, H, Hs, E_r, r1 = c["d"], c["H"], c["Hs"], c["E_r"], _projections(c)
        resident = np.zeros(c["E"], np.uint8)
        resident[D.r.choice(c["E"], E_r, replace=False)] = 1
        s = dict(case=c, x=D.normal(c["T"], d, dtype=dt),
                 w_router=D.normal(c["E"], d, std=0.02, dtype=dt),
                 bias=D.normal(c["E"], std=0.1) if c["bias"] else None,
                 resident=torch.from_numpy(resident).cuda())
        for name, n, rows, cols in (("w_gate_up", E_r, r1 * H, d), ("w_down", E_r, d, H),
                                    ("shared_gate_up", 1, r1 * Hs, d), ("shared_down", 1, d, Hs)):
            if rows and cols:
                s[name] = (D.mx(n, rows, cols) if c["weights"] == "mxfp4"
                           else D.normal(n, rows, cols, std=0.02, dtype=dt))
        return s
    if c["family"] == "quant":
        # rows of uneven scale, so that the blocks' scales span a range
        x = D.normal(c["rows"], c["cols"]) * torch.exp2(4 * D.normal(c["rows"], 1))
        return dict(case=c, x=x.to(dt))
    n, E_r = c["n"], c["E_r"]
    p = np.arange(1, E_r + 1) ** (-1.2 if c["skew"] else 0.0)
    sizes = D.r.multinomial(n, D.r.permutation(p / p.sum()))
    off = np.concatenate([[0], np.cumsum(sizes)])
    return dict(case=c, x=D.normal(n, c["d"], dtype=dt), sizes=[int(v) for v in sizes],
                offsets=torch.from_numpy(off.astype(np.int32)).cuda(),
                w_gate_up=D.mx(E_r, _projections(c) * c["H"], c["d"]),
                w_down=D.mx(E_r, c["d"], c["H"]))


# ------------------------------------------------------------------ the framework's calls
def _own_norm(s):
    from paper_2606_19025_amd.layer import LayerNorm

    c = s["case"]
    if "own" not in s:
        s["own"] = LayerNorm(c["T"], c["d"], dtype=DTYPES[c["dtype"]], bias=c["bias"], eps=EPS)
    N, out = s["own"], {}
    if c["way"] != "bwd":
        N.forward(s["x"], s["w"], s["b"])
        out.update(y=N.y, mean=N.mean, rstd=N.rstd)
    if c["way"] == "fwd":
        return out
    stats = dict(mean=s["mean"], rstd=s["rstd"]) if c["way"] == "bwd" else {}
    N.backward(s["dy"], s["x"], s["w"], dres=s["dres"], **stats)
    out.update(dx=N.dx, dw=N.dw)
    if c["bias"]:
        out["db"] = N.db
    return out


def _own_few(s):
    from paper_2606_19025_amd.layer import InferenceMoELayer

    c = s["case"]
    if "own" not in s:
        s["own"] = InferenceMoELayer(
            c["k"], s["resident"], s["w_router"], s["w_gate_up"], s["w_down"],
            router_bias=s["bias"], shared_gate_up=s.get("shared_gate_up"),
            shared_down=s.get("shared_down"), gate=c["gate"], expert=c["expert"])
    L = s["own"]
    y = L.few(s["x"])
    return dict(y=y, logits=L.logits, idx=L.topk_idx, w=L.topk_w, local=L.topk_local)


def _own_quant(s):
    from paper_2606_19025_amd.layer import mxfp4_dequantize, mxfp4_quantize

    s["q"] = mxfp4_quantize(s["x"], out=s.get("q"))
    s["v"] = mxfp4_dequantize(*s["q"], DTYPES[s["case"]["dtype"]], out=s.get("v"))
    return dict(values=s["v"])


def _own_mxffn(s):
    from paper_2606_19025_amd.layer import MxFFN

    c = s["case"]
    if "own" not in s:
        s["own"] = MxFFN(c["n"], s["w_gate_up"], s["w_down"], expert=c["expert"])
    return dict(y=s["own"].forward(s["x"], s["offsets"]))


# ------------------------------------------------------------------ the plain forms
def _plain_norm(s):
    c, w, out = s["case"], s["w"], {}
    dt, x = DTYPES[c["dtype"]], s["x"].float()
    if c["way"] == "bwd":
        mean, rstd = s["mean"], s["rstd"]
        xh = (x - mean[:, None]) * rstd[:, None]
    else:
        mean = x.mean(dim=1)
        xc = x - mean[:, None]
        rstd = ((xc * xc).mean(dim=1) + EPS).rsqrt()
        xh = xc * rstd[:, None]
        y = xh * w
        if c["bias"]:
            y = y + s["b"]
        out.update(y=y.to(dt), mean=mean, rstd=rstd)
    if c["way"] == "fwd":
        return out
    dy = s["dy"].float()
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    out.update(dx=dx.to(dt), dw=(dy * xh).sum(dim=0))
    if c["bias"]:
        out["db"] = dy.sum(dim=0)
    return out


def _weights(w):
    """32-bit [n, rows, cols] of plain or MXFP4 weights."""
    if isinstance(w, tuple):
        codes, scales = w
        return _mx_unpack(codes.flatten(0, 1), scales.flatten(0, 1)).view(*codes.shape[:2], -1)
    return w.float()


def _act(a, expert):
    if expert == "silu":
        return a * torch.sigmoid(a)
    g, u = a.chunk(2, dim=-1)
    return g * torch.sigmoid(g) * u


def _route(c, z, resident):
    """(experts, gate weights, local ids) of the k largest logits, the lower id first among equals."""
    order = torch.sort(z, dim=1, descending=True, stable=True)
    idx, top = order.indices[:, : c["k"]], order.values[:, : c["k"]]
    if c["gate"] == "softmax_topk":
        w = torch.softmax(top, dim=1)
    elif c["gate"] == "softmax":
        w = torch.softmax(z, dim=1).gather(1, idx)
    else:
        w = torch.sigmoid(top)
    local = torch.where(resident != 0, torch.cumsum(resident.long(), 0) - 1, -1)[idx]
    return idx, w, local


def _plain_few(s):
    c, dt, x = s["case"], DTYPES[s["case"]["dtype"]], s["x"].float()
    T, d, k, E_r = c["T"], c["d"], c["k"], c["E_r"]
    z = s["x"].double() @ s["w_router"].double().T
    if s["bias"] is not None:
        z = z + s["bias"].double()
    idx, w, local = _route(c, z, s["resident"])
    gate = torch.where(local >= 0, w, 0.0).float()
    at = local.clamp(min=0)
    if T * k <= E_r:
        # fewer routes than experts: each route's own weights
        pick = at.reshape(-1)
        if c["weights"] == "mxfp4":
            wgu, wd = (_weights((q[pick], sc[pick])) for q, sc in (s["w_gate_up"], s["w_down"]))
        else:
            wgu, wd = s["w_gate_up"][pick].float(), s["w_down"][pick].float()
        h = _act(torch.matmul(wgu, x.repeat_interleave(k, 0)[:, :, None])[..., 0], c["expert"])
        y = torch.matmul(wd, h[:, :, None]).view(T, k, d)
        y = (y * gate[:, :, None]).sum(dim=1)
    else:
        # every expert on every token, under gates that are zero off the routes
        full = torch.zeros(T, E_r, device=x.device).scatter_add_(1, at, gate)
        wgu, wd = _weights(s["w_gate_up"]), _weights(s["w_down"])
        h = _act((x @ wgu.flatten(0, 1).T).view(T, E_r, -1), c["expert"]) * full[:, :, None]
        y = h.flatten(1) @ wd.transpose(1, 2).reshape(-1, d)
    if c["Hs"]:
        h = _act(x @ _weights(s["shared_gate_up"])[0].T, c["expert"])
        y = y + h @ _weights(s["shared_down"])[0].T
    return dict(y=y.to(dt), logits=z.float(), idx=idx.int(), w=w.float(), local=local.int())


def _plain_mxffn(s):
    x = _mx_values(*_mx_blocks(s["x"]))
    wgu, wd = _weights(s["w_gate_up"]), _weights(s["w_down"])
    # a product per expert and projection
    a = torch.cat([r @ w.T for r, w in zip(x.split(s["sizes"]), wgu)])
    h = _mx_values(*_mx_blocks(_act(a, s["case"]["expert"])))
    return dict(y=torch.cat([r @ w.T for r, w in zip(h.split(s["sizes"]), wd)]).to(torch.bfloat16))


def run(s):
    family = s["case"]["family"]
    if own:
        return {"norm": _own_norm, "few": _own_few, "quant": _own_quant,
                "mxffn": _own_mxffn}[family](s)
    if family == "norm":
        return _plain_norm(s)
    if family == "few":
        return _plain_few(s)
    if family == "quant":
        return dict(values=_mx_values(*_mx_blocks(s["x"])).to(DTYPES[s["case"]["dtype"]]))
    return _plain_mxffn(s)


# ------------------------------------------------------------------ exact
def _pow2(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_mx(v):
    """Rows of 64-bit values rounded to MXFP4: per block of 32 the exponent of the largest
    magnitude (from its logarithm's integer part, by frexp), then the nearest value of the
    grid, found by distance (the even code where two are as near)."""
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(top).exponent - 1 - 2).clamp(min=-127)
    a = b * _pow2(-e)
    grid = torch.tensor(E2M1, dtype=torch.float64, device=v.device)
    up = torch.bucketize(a.abs(), grid).clamp(max=7)
    lo = (up - 1).clamp(min=0)
    m = a.abs().clamp(max=6.0)
    near_lo, near_hi = m - grid[lo], grid[up] - m
    take_lo = (near_lo < near_hi) | ((near_lo == near_hi) & (lo % 2 == 0))
    return (torch.where(take_lo, grid[lo], grid[up]) * torch.sign(a) * _pow2(e)).reshape(v.shape)


def _exact_weights(w):
    if not isinstance(w, tuple):
        return w.double()
    codes, scales = w
    n, rows, half = codes.shape
    nib = torch.empty(n, rows, 2 * half, dtype=torch.long, device=codes.device)
    nib[..., 0::2], nib[..., 1::2] = codes % 16, codes // 16
    # E2M1: 1 sign, 2 exponent, 1 mantissa bit; exponent 0 holds 0 and 0.5
    sign, ex, man = 1 - 2 * (nib // 8), nib // 2 % 4, (nib % 2).double()
    mag = torch.where(ex == 0, man / 2, (1 + man / 2) * _pow2(ex - 1))
    e = scales[..., : 2 * half // 32].long().repeat_interleave(32, dim=2) - 127
    return sign * mag * _pow2(e)


def _exact_act(a, expert):
    H = a.shape[-1] if expert == "silu" else a.shape[-1] // 2
    g = a[..., :H]
    h = g / (1 + torch.exp(-g))
    return h if expert == "silu" else h * a[..., H:]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["family"] == "norm":
        x, w, out = s["x"].double(), s["w"].double(), {}
        d = c["d"]
        mu = x.sum(dim=1, keepdim=True) / d
        r = 1 / torch.sqrt(((x - mu) ** 2).sum(dim=1, keepdim=True) / d + EPS)
        if c["way"] != "bwd":
            y = (x - mu) * r * w + (s["b"].double() if c["bias"] else 0.0)
            out.update(y=y, mean=mu[:, 0], rstd=r[:, 0])
        else:
            mu, r = s["mean"].double()[:, None], s["rstd"].double()[:, None]
        if c["way"] == "fwd":
            return out
        dy, xh = s["dy"].double(), (x - mu) * r
        g = dy * w
        dx = r * g - r / d * g.sum(dim=1, keepdim=True) - r / d * xh * (g * xh).sum(dim=1, keepdim=True)
        out.update(dx=dx if s["dres"] is None else dx + s["dres"].double(), dw=(dy * xh).sum(dim=0))
        if c["bias"]:
            out["db"] = dy.sum(dim=0)
        return out
    if c["family"] == "quant":
        return dict(values=_exact_mx(s["x"].double()))
    if c["family"] == "mxffn":
        x, out, at = _exact_mx(s["x"].double()), [], 0
        for g, n in enumerate(s["sizes"]):
            wgu, wd = (_exact_weights((q[g:g + 1], sc[g:g + 1]))[0]
                       for q, sc in (s["w_gate_up"], s["w_down"]))
            h = _exact_mx(_exact_act(x[at:at + n] @ wgu.T, c["expert"]))
            out.append(h @ wd.T)
            at += n
        return dict(y=torch.cat(out))
    x = s["x"].double()
    z = x @ s["w_router"].double().T + (s["bias"].double() if s["bias"] is not None else 0.0)
    resident = s["resident"].tolist()
    slot = {e: sum(resident[:e]) for e in range(c["E"]) if resident[e]}
    y = torch.zeros_like(x)
    w = torch.zeros(c["T"], c["k"], dtype=torch.float64, device=x.device)
    rows = z.tolist()
    routes = {}
    for t, row in enumerate(rows):
        ids = sorted(range(c["E"]), key=lambda e: (-row[e], e))[: c["k"]]
        top = [math.exp(row[e] - row[ids[0]]) for e in ids]
        total = sum(top) if c["gate"] == "softmax_topk" else sum(math.exp(v - row[ids[0]]) for v in row)
        for j, e in enumerate(ids):
            gate = 1 / (1 + math.exp(-row[e])) if c["gate"] == "sigmoid" else top[j] / total
            w[t, j] = gate
            if e in slot:
                routes.setdefault(slot[e], []).append((t, gate))
    for r, who in routes.items():
        wgu, wd = (_exact_weights(tuple(q[r:r + 1] for q in v) if isinstance(v, tuple) else v[r:r + 1])[0]
                   for v in (s["w_gate_up"], s["w_down"]))
        ts = torch.tensor([t for t, _ in who], device=x.device)
        gates = torch.tensor([g for _, g in who], dtype=torch.float64, device=x.device)
        y.index_add_(0, ts, _exact_act(x[ts] @ wgu.T, c["expert"]) @ wd.T * gates[:, None])
    if c["Hs"]:
        h = _exact_act(x @ _exact_weights(s["shared_gate_up"])[0].T, c["expert"])
        y += h @ _exact_weights(s["shared_down"])[0].T
    return dict(y=y, logits=z, idx=None, w=w, local=None)


# ------------------------------------------------------------------ work
def _mx_bytes(rows, cols):
    return rows * (cols // 2 + cols // 32)


def work(case):
    c = case
    if c["family"] == "norm":
        n, e, s = c["T"] * c["d"], SIZE[c["dtype"]], 8 * c["T"]
        small = 4 * c["d"] * (2 if c["bias"] else 1)
        fwd, bwd = 2 * e * n + s + small, (4 if c["res"] else 3) * e * n + s + small
        x_once = e * n if c["way"] == "both" else 0  # x is one input of the pass
        return dict(bytes=(fwd if c["way"] != "bwd" else 0) + (bwd if c["way"] != "fwd" else 0) - x_once,
                    flops=(8 * n if c["way"] != "bwd" else 0) + (14 * n if c["way"] != "fwd" else 0))
    if c["family"] == "quant":
        n, q = c["rows"] * c["cols"], _mx_bytes(c["rows"], c["cols"])
        return dict(bytes=2 * SIZE[c["dtype"]] * n + 2 * q, flops=3 * n)
    r1, d, H = _projections(c), c["d"], c["H"]
    if c["family"] == "mxffn":
        active = c["E_r"] * (1 - (1 - 1 / c["E_r"]) ** c["n"]) if not c["skew"] else min(c["E_r"], c["n"])
        w = active * (_mx_bytes(r1 * H, d) + _mx_bytes(d, H))
        return dict(bytes=w + 4 * c["n"] * d, flops=2 * c["n"] * d * H * (r1 + 1))
    T, e = c["T"], SIZE[c["dtype"]]
    # experts that T tokens of k routes each are expected to reach
    active = c["E_r"] * (1 - (1 - c["k"] / c["E"]) ** T)

    def block(h):
        return (_mx_bytes(r1 * h, d) + _mx_bytes(d, h) if c["weights"] == "mxfp4"
                else e * (r1 + 1) * d * h) if h else 0

    routes = T * c["k"] * c["E_r"] / c["E"]
    return dict(bytes=active * block(H) + block(c["Hs"]) + e * (c["E"] * d + 2 * T * d)
                + T * (4 * c["E"] + 12 * c["k"]),
                flops=2 * d * (T * c["E"] + (r1 + 1) * (routes * H + T * c["Hs"])))
