"""Performance cases of the operators that complete a worker's training step.

Each case is one pass through an operator, as a training or evaluation loop
calls it:

  xent    softmax cross entropy of a linear head over a vocabulary, without the
          logits being kept: the losses, or the losses and both gradients
  block   the norms and the residual sum around a block (x' = x + a g norm(f),
          u = norm(x')): forward or backward
  clip    the norm of all gradients together and the gradients clipped by it
  adamw   the same norm, and AdamW on all parameters with clipped gradients

With ``own`` false ``run`` computes the operators in elementary torch
operations, in 32 bits (sums of squares over all gradients in 64); with ``own``
true it calls the framework.  ``exact`` computes them in 64 bits from their
definitions.  Activations are ~ N(0, 1), weights ~ N(0, 0.02), as in
``paper_2606_19025_amd.inputs``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5                                  # of the norms
LR, BETA1, BETA2, ADAM_EPS = 3e-4, 0.9, 0.95, 1e-8
STEP = 7                                    # the optimiser's step count


def _xent(name, way, N, d, V, dtype="bf16", ignored=0.0, mean=True, scale=1.0, z_coef=0.0):
    return dict(name=name, family="xent", way=way, N=N, d=d, V=V, dtype=dtype, ignored=ignored,
                mean=mean, scale=scale, z_coef=z_coef)


def _block(name, way, T, d, dtype="bf16", post=True, gate="none", bias=True, scale=1.0):
    return dict(name=name, family="block", way=way, T=T, d=d, dtype=dtype, post=post, gate=gate,
                bias=bias, scale=scale)


def _tensors(name, family, count, small, large, bf16=0.0, params=0, decay=0.0, max_norm=1.0):
    """count tensors of small to large values each (their logarithms even), a share bf16 of them in
    bf16; params > 0: together about that many values."""
    return dict(name=name, family=family, count=count, small=small, large=large, bf16=bf16,
                params=params, decay=decay, max_norm=max_norm)


def listed():
    return [
        # a few tokens scored against a whole vocabulary: the weights' stream
        _xent("xent-eval-few-bf16", "fwd", 24, 2048, 49152),
        # the tiny fp32 layer's model: launches and latency
        _xent("xent-tiny-f32", "step", 256, 64, 1000, dtype="f32"),
        # the loss of the fine-grained workload's training step
        _xent("xent-step-fine-bf16", "step", 8192, 2048, 49152),
        # a last, ragged micro-batch with padding and weights of its own for every token,
        # a vocabulary of odd size, the logits' scale of a transferred width and a penalty on lse
        _xent("xent-step-odd-bf16", "step", 1531, 768, 50003, ignored=0.3, mean=False, scale=0.5,
              z_coef=1e-4),
        # between two blocks for one generated token: latency alone
        _block("block-fwd-one-bf16", "fwd", 1, 2048),
        # between two blocks of the fine-grained workload
        _block("block-fwd-fine-bf16", "fwd", 8192, 2048, scale=0.25),
        # the large workload's backward, with a learned gate for each channel
        _block("block-bwd-large-bf16", "bwd", 16384, 4096, gate="channel"),
        # an fp32 run on a last, ragged micro-batch of an odd width, a gate for each token, no biases
        _block("block-bwd-odd-f32", "bwd", 3001, 520, dtype="f32", gate="token", bias=False),
        # the gradients of the fine-grained layer: few tensors, most of them large
        _tensors("clip-fine-f32", "clip", 9, 1 << 17, 1 << 27, params=156_000_000),
        # the dense part of a model: many small tensors, some of them in bf16
        _tensors("clip-many-mixed", "clip", 300, 64, 1 << 17, bf16=0.3),
        # the fine-grained layer's parameters
        _tensors("adamw-fine-f32", "adamw", 9, 1 << 17, 1 << 27, params=156_000_000),
        # norms, biases, routers and a few matrices, with weight decay
        _tensors("adamw-many-mixed", "adamw", 200, 64, 1 << 18, bf16=0.3, decay=0.1),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of step between lo and hi, uniform over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    family = rng.choice(["xent", "xent", "xent", "block", "block", "clip", "adamw"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if family == "xent":
        way = rng.choice(["fwd", "step", "step"])
        d, V = _log(rng, 64, 4096, 64), _log(rng, 100, 65536)
        # at most a third of the largest listed case's operations (fp32: a thirtieth)
        N = max(1, min(_log(rng, 1, 8192), int((2.7e11 if dtype == "bf16" else 2.7e10) / (d * V))))
        c = _xent("", way, N, d, V, dtype, rng.choice([0.0, 0.1, 0.5]), rng.random() < 0.5,
                  rng.choice([1.0, 1.0, 0.5]), rng.choice([0.0, 0.0, 1e-4]))
    elif family == "block":
        T, d = _log(rng, 1, 16384), _log(rng, 64, 8192, 8)
        T = max(1, min(T, (1 << 26) // d))
        c = _block("", rng.choice(["fwd", "bwd"]), T, d, dtype, rng.random() < 0.8,
                   rng.choice(["none", "channel", "token"]), rng.random() < 0.7,
                   rng.choice([1.0, 0.25]))
    else:
        small, large = _log(rng, 1, 4096), _log(rng, 4096, 1 << 24)
        count = max(1, min(_log(rng, 1, 400), (1 << 28) // large))
        c = _tensors("", family, count, small, large, rng.choice([0.0, 0.3, 1.0]), 0,
                     rng.choice([0.0, 0.1]), rng.choice([1.0, 1e6]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
class _Draw:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))
        self.r = np.random.default_rng(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        out = torch.empty(*shape, dtype=dtype, device="cuda")
        return out.normal_(mean, std, generator=self.g)

    def uniform(self, *shape):
        return torch.empty(*shape, device="cuda").uniform_(generator=self.g)


def _stats(x):
    """Mean and reciprocal deviation of rows, in 64 bits."""
    x = x.double()
    mean = x.mean(dim=1)
    return mean, (((x - mean[:, None]) ** 2).mean(dim=1) + EPS).rsqrt()


def prepare(case, seed):
    c, D = case, _Draw(seed)
    if c["family"] == "xent":
        N, d, V, dt = c["N"], c["d"], c["V"], DTYPES[c["dtype"]]
        # words by a power law; hidden states that lean towards their label's weights
        labels = (D.uniform(N) ** 3 * V).long().clamp_(max=V - 1)
        w = D.normal(V, d, std=0.02, dtype=dt)
        x = (D.normal(N, d) + 2.0 * w[labels].float()).to(dt)
        if c["ignored"]:
            labels = torch.where(D.uniform(N) < c["ignored"], -1, labels)
        s = dict(case=c, x=x, w=w, labels=labels.int(), dloss=None)
        if not c["mean"]:
            s["dloss"] = D.uniform(N) / N
        return s
    if c["family"] == "block":
        T, d, dt = c["T"], c["d"], DTYPES[c["dtype"]]
        gate = {"none": lambda: None, "channel": lambda: D.normal(d, std=0.2, mean=0.5),
                "token": lambda: D.uniform(T)}[c["gate"]]()
        # a residual stream (a row mean of its own, features of uneven scale) and a block's output
        s = dict(case=c, f=D.normal(T, d, std=0.3, dtype=dt), gate=gate,
                 x=(D.normal(T, d) * D.normal(d, std=0.3).exp_() + D.normal(T, 1, std=0.5)).to(dt),
                 pre_w=D.normal(d, std=0.1, mean=1.0), pre_b=None, post_w=None, post_b=None)
        if c["post"]:
            s["post_w"] = D.normal(d, std=0.1, mean=1.0)
        if c["bias"]:
            s["pre_b"] = D.normal(d, std=0.1)
            if c["post"]:
                s["post_b"] = D.normal(d, std=0.1)
        if c["way"] == "bwd":  # what the forward left (x is the residual stream behind the sum)
            s["du"], s["dres"] = D.normal(T, d, dtype=dt), D.normal(T, d, dtype=dt)
            s["pre_mean"], s["pre_rstd"] = (v.float() for v in _stats(s["x"]))
            if c["post"]:
                s["post_mean"], s["post_rstd"] = (v.float() for v in _stats(s["f"]))
        return s
    # gradients of uneven scale; a case's sizes and types are its own, whatever the seed
    n = c["count"]
    r = np.random.default_rng([n, c["small"], c["large"]])
    sizes = np.exp(r.uniform(math.log(c["small"]), math.log(c["large"]), n))
    if c["params"]:
        sizes *= c["params"] / sizes.sum()
    sizes = [max(1, int(v)) for v in sizes]
    bf16 = r.random(n) < c["bf16"]
    scales = np.exp(D.r.normal(-4.0, 1.0, n))
    grads = [D.normal(m, std=float(e), dtype=torch.bfloat16 if b else torch.float32)
             for m, e, b in zip(sizes, scales, bf16)]
    s = dict(case=c, grads=grads)
    if c["family"] == "clip":
        # clipped gradients, as a step keeps them: one buffer of each type, pieces from 16-byte borders
        at = np.cumsum([0] + [(m + 7) // 8 * 8 for m in sizes])
        flat = {dt: torch.zeros(int(at[-1]), dtype=dt, device="cuda")
                for dt in {g.dtype for g in grads}}
        s.update(flat=flat, out=[flat[g.dtype][int(a): int(a) + g.numel()]
                                 for g, a in zip(grads, at)])
        return s
    # parameters and moments in flat buffers, pieces from 16-byte borders
    at = [int(a) for a in np.cumsum([0] + [(m + 7) // 8 * 8 for m in sizes])]
    piece = lambda t: [t[a: a + m] for a, m in zip(at, sizes)]
    s["flat"] = dict(theta=D.normal(at[-1], std=0.02), m=D.normal(at[-1], std=0.01),
                     v=D.normal(at[-1], std=0.01).square_())
    s["flat"]["low"] = s["flat"]["theta"].bfloat16()
    s.update({k: piece(t) for k, t in s["flat"].items()})
    return s


# ------------------------------------------------------------------ the framework's calls
def _own_xent(s):
    from paper_2606_19025_amd.train import LinearCrossEntropy

    c = s["case"]
    if "own" not in s:
        s["own"] = LinearCrossEntropy(c["N"], c["d"], c["V"], dtype=DTYPES[c["dtype"]],
                                      scale=c["scale"], z_coef=c["z_coef"],
                                      dw_dtype=DTYPES[c["dtype"]])
    L = s["own"]
    L.forward(s["x"], s["w"], s["labels"])
    out = dict(loss=L.loss, lse=L.lse, total=L.total)
    if c["way"] == "step":
        L.backward(s["x"], s["w"], s["labels"], dloss=s["dloss"])
        out.update(dx=L.dx, dw=L.dw)
    return out


def _own_block(s):
    from paper_2606_19025_amd.layer import BlockNorm

    c = s["case"]
    if "own" not in s:
        s["own"] = BlockNorm(c["T"], c["d"], dtype=DTYPES[c["dtype"]], post=c["post"],
                             gate=None if c["gate"] == "none" else c["gate"], bias=c["bias"],
                             scale=c["scale"], eps=EPS)
    K = s["own"]
    if c["way"] == "fwd":
        K.forward(s["x"], s["f"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"])
        out = dict(x=K.x, u=K.u, pre_mean=K.pre_mean, pre_rstd=K.pre_rstd)
        if c["post"]:
            out.update(post_mean=K.post_mean, post_rstd=K.post_rstd)
        return out
    stats = {k: s[k] for k in ("pre_mean", "pre_rstd", "post_mean", "post_rstd") if k in s}
    K.backward(s["du"], s["f"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], dres=s["dres"],
               x=s["x"], **stats)
    out = dict(dx=K.dx, df=K.df, d_pre_w=K.d_pre_weight)
    if c["bias"]:
        out["d_pre_b"] = K.d_pre_bias
    if c["post"]:
        out["d_post_w"] = K.d_post_weight
        if c["bias"]:
            out["d_post_b"] = K.d_post_bias
    if c["gate"] != "none":
        out["d_gate"] = K.d_gate
    return out


def _flat_outputs(s):
    return {str(k).replace("torch.", ""): v for k, v in s["flat"].items()}


def _own_clip(s):
    from paper_2606_19025_amd.train import GradClipper

    if "own" not in s:
        s["own"] = GradClipper(s["grads"], s["case"]["max_norm"], out=s["out"])
    norm = s["own"].clip()
    return dict(norm=norm, **_flat_outputs(s))


def _own_adamw(s):
    from paper_2606_19025_amd.train import AdamW

    c = s["case"]
    if "own" not in s:
        s["own"] = AdamW(s["theta"], s["grads"], s["m"], s["v"], theta_bf16=s["low"],
                         max_norm=c["max_norm"], betas=(BETA1, BETA2), eps=ADAM_EPS,
                         weight_decay=c["decay"])
    norm = s["own"].step(STEP, LR)
    return dict(norm=norm, **_flat_outputs(s))


# ------------------------------------------------------------------ the plain forms
def _plain_xent(s):
    c, x, w, y = s["case"], s["x"].float(), s["w"].float(), s["labels"].long()
    z = (x @ w.T) * c["scale"]
    top = z.amax(dim=1, keepdim=True)
    p = (z - top).exp()
    total = p.sum(dim=1, keepdim=True)
    lse = (total.log() + top)[:, 0]
    counted = y >= 0
    at = y.clamp(min=0)[:, None]
    loss = lse - z.gather(1, at)[:, 0] + c["z_coef"] * lse * lse
    loss, lse = torch.where(counted, loss, 0.0), torch.where(counted, lse, 0.0)
    n = counted.sum().float()
    out = dict(loss=loss, lse=lse, total=torch.stack([loss.sum(), n]))
    if c["way"] == "fwd":
        return out
    g = s["dloss"] if s["dloss"] is not None else torch.ones_like(lse) / n.clamp(min=1)
    g = torch.where(counted, g * c["scale"], 0.0)
    p *= (g * (1 + 2 * c["z_coef"] * lse))[:, None] / total
    p.scatter_add_(1, at, -g[:, None])
    out.update(dx=(p @ w).to(s["x"].dtype), dw=(p.T @ x).to(s["w"].dtype))
    return out


def _norm(x, mean, rstd):
    return (x - mean[:, None]) * rstd[:, None]


def _moments(x):
    mean = x.mean(dim=1)
    xc = x - mean[:, None]
    return mean, ((xc * xc).mean(dim=1) + EPS).rsqrt()


def _norm_bwd(g, xh, rstd):
    return rstd[:, None] * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))


def _weighted(n, w, b):
    if w is None:
        return n
    return n * w if b is None else n * w + b


def _gate(s, a):
    """The factor a g of the block's output: [T, 1], [d] or a number."""
    g = s["gate"]
    if g is None:
        return a
    return a * g[:, None] if s["case"]["gate"] == "token" else a * g


def _plain_block(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    x, f = s["x"].float(), s["f"].float()
    if c["way"] == "fwd":
        out, n = {}, f
        if c["post"]:
            mean, rstd = _moments(f)
            n = _weighted(_norm(f, mean, rstd), s["post_w"], s["post_b"])
            out.update(post_mean=mean, post_rstd=rstd)
        x = (x + _gate(s, c["scale"]) * n).to(dt)
        mean, rstd = _moments(x.float())
        u = _weighted(_norm(x.float(), mean, rstd), s["pre_w"], s["pre_b"])
        out.update(x=x, u=u.to(dt), pre_mean=mean, pre_rstd=rstd)
        return out
    du = s["du"].float()
    xh = _norm(x, s["pre_mean"], s["pre_rstd"])
    G = s["dres"].float() + _norm_bwd(du * s["pre_w"], xh, s["pre_rstd"])
    out = dict(dx=G.to(dt), d_pre_w=(du * xh).sum(dim=0))
    if c["bias"]:
        out["d_pre_b"] = du.sum(dim=0)
    dn = G * _gate(s, c["scale"])
    n = f
    if c["post"]:
        fh = _norm(f, s["post_mean"], s["post_rstd"])
        n = _weighted(fh, s["post_w"], s["post_b"])
        out["d_post_w"] = (dn * fh).sum(dim=0)
        if c["bias"]:
            out["d_post_b"] = dn.sum(dim=0)
        dn = _norm_bwd(dn * s["post_w"], fh, s["post_rstd"])
    out["df"] = dn.to(dt)
    if c["gate"] != "none":
        out["d_gate"] = c["scale"] * (G * n).sum(dim=1 if c["gate"] == "token" else 0)
    return out


def _plain_norm(s):
    """[norm, scale] of all gradients."""
    squares = torch.stack([g.double().square().sum() for g in s["grads"]])
    norm = squares.sum().sqrt().float()
    return torch.stack([norm, (s["case"]["max_norm"] / norm).clamp(max=1.0)])


def _plain_clip(s):
    norm = _plain_norm(s)
    [o.copy_((g.float() * norm[1]).to(g.dtype)) for g, o in zip(s["grads"], s["out"])]
    return dict(norm=norm, **_flat_outputs(s))


def _adamw(th, g, m, v, low, scale, decay):
    g = g.float() * scale
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    den = (v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS
    th.sub_(LR * (m / (1 - BETA1 ** STEP) / den + decay * th))
    low.copy_(th)


def _plain_adamw(s):
    norm = _plain_norm(s)
    [_adamw(*t, norm[1], s["case"]["decay"])
     for t in zip(s["theta"], s["grads"], s["m"], s["v"], s["low"])]
    return dict(norm=norm, **_flat_outputs(s))


_OWN = dict(xent=_own_xent, block=_own_block, clip=_own_clip, adamw=_own_adamw)
_PLAIN = dict(xent=_plain_xent, block=_plain_block, clip=_plain_clip, adamw=_plain_adamw)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["family"]](state)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    if c["family"] == "xent":
        N, d, V, s = c["N"], c["d"], c["V"], SIZE[c["dtype"]]
        step = c["way"] == "step"
        return {"bytes": (N * d + V * d) * s * (2 if step else 1) + 12 * N,
                "flops": (6 if step else 2) * N * d * V}
    if c["family"] == "block":
        T, d, s = c["T"], c["d"], SIZE[c["dtype"]]
        if c["way"] == "fwd":
            return {"bytes": 4 * T * d * s + 16 * T + 16 * d, "flops": 20 * T * d}
        return {"bytes": 6 * T * d * s + 16 * T + 32 * d, "flops": 40 * T * d}
    # the mean size of a tensor, as the sizes are drawn
    lo, hi = c["small"], c["large"]
    n = c["params"] or c["count"] * ((hi - lo) / math.log(hi / lo) if hi > lo else lo)
    g = 4 - 2 * c["bf16"]
    if c["family"] == "clip":
        return {"bytes": int(n * 3 * g), "flops": int(3 * n)}
    return {"bytes": int(n * (2 * g + 24 + 2)), "flops": int(16 * n)}


# ------------------------------------------------------------------ in 64 bits
def _exact_xent(s):
    c, y = s["case"], s["labels"].long()
    x, w = s["x"].double(), s["w"].double()
    z = x.matmul(w.t()).mul_(c["scale"])
    keep = y.ge(0)
    lse = torch.logsumexp(z, dim=1) * keep  # tokens that do not count have none
    rows = keep.nonzero()[:, 0]
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - z[rows, y[rows]] + c["z_coef"] * lse[rows] ** 2
    count = rows.numel()
    out = dict(loss=loss, lse=lse,
               total=torch.stack([loss.sum(), torch.tensor(float(count), device=z.device).double()]))
    if c["way"] == "fwd":
        return out
    # d loss_t / d z = (1 + 2 z_coef lse) softmax(z) - onehot
    dz = z.sub_(lse[:, None]).exp_().mul_((1 + 2 * c["z_coef"] * lse)[:, None])
    dz[rows, y[rows]] -= 1
    up = s["dloss"].double() if s["dloss"] is not None else torch.full_like(lse, 1.0 / max(count, 1))
    dz.mul_((up * keep * c["scale"])[:, None])
    out.update(dx=dz.matmul(w), dw=dz.t().matmul(x))
    return out


def _exact_block(s):
    c = s["case"]
    dbl = {k: v.double() if torch.is_tensor(v) else v for k, v in s.items()}
    x, f, d = dbl["x"], dbl["f"], c["d"]
    g = dbl["gate"]
    ag = c["scale"] * (torch.ones(d, device=x.device).double()[None] if g is None
                       else g[:, None] if c["gate"] == "token" else g[None])
    affine = lambda h, w, b: h if w is None else h * w + (0 if b is None else b)
    if c["way"] == "fwd":
        out, n = {}, f
        if c["post"]:
            pm, pr = _stats(f)
            out.update(post_mean=pm, post_rstd=pr)
            n = affine((f - pm[:, None]) * pr[:, None], dbl["post_w"], dbl["post_b"])
        x = x + ag * n
        # the stream is kept in its own type, and the next norm reads that
        kept = x.to(s["x"].dtype).double()
        mean, r = _stats(kept)
        u = affine((kept - mean[:, None]) * r[:, None], dbl["pre_w"], dbl["pre_b"])
        out.update(x=x, u=u, pre_mean=mean, pre_rstd=r)
        return out
    du = dbl["du"]
    r = dbl["pre_rstd"][:, None]
    xh = (x - dbl["pre_mean"][:, None]) * r
    gx = du * dbl["pre_w"]
    G = dbl["dres"] + r * (gx - gx.sum(1, keepdim=True) / d - xh * ((gx * xh).sum(1, keepdim=True) / d))
    out = dict(dx=G, d_pre_w=(du * xh).sum(0))
    if c["bias"]:
        out["d_pre_b"] = du.sum(0)
    dn, n = G * ag, f
    if c["post"]:
        q = dbl["post_rstd"][:, None]
        fh = (f - dbl["post_mean"][:, None]) * q
        n = affine(fh, dbl["post_w"], dbl["post_b"])
        out["d_post_w"] = (dn * fh).sum(0)
        if c["bias"]:
            out["d_post_b"] = dn.sum(0)
        h = dn * dbl["post_w"]
        dn = q * (h - h.sum(1, keepdim=True) / d - fh * ((h * fh).sum(1, keepdim=True) / d))
    out["df"] = dn
    if c["gate"] != "none":
        out["d_gate"] = (c["scale"] * G * n).sum(1 if c["gate"] == "token" else 0)
    return out


def _exact_tensors(s):
    c = s["case"]
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grads"]))
    scale = min(1.0, c["max_norm"] / norm)
    out = dict(norm=torch.tensor([norm, scale], dtype=torch.float64))
    flat = {k: t.double() for k, t in _flat_outputs(s).items()}
    if c["family"] == "clip":
        name = {g.dtype: str(g.dtype).replace("torch.", "") for g in s["grads"]}
        first = {dt: t.data_ptr() for dt, t in s["flat"].items()}
        for g, o in zip(s["grads"], s["out"]):
            a = (o.data_ptr() - first[g.dtype]) // g.element_size()
            flat[name[g.dtype]][a: a + g.numel()] = scale * g.double()
        return dict(out, **flat)
    first = s["flat"]["theta"].data_ptr()
    for th, g in zip(s["theta"], s["grads"]):
        at = slice((th.data_ptr() - first) // 4, (th.data_ptr() - first) // 4 + g.numel())
        q = scale * g.double()
        m = BETA1 * flat["m"][at] + (1 - BETA1) * q
        v = BETA2 * flat["v"][at] + (1 - BETA2) * q * q
        mh, vh = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
        t = flat["theta"][at]
        flat["m"][at], flat["v"][at] = m, v
        flat["theta"][at] = t - LR * (mh / (vh.sqrt() + ADAM_EPS) + c["decay"] * t)
        flat["low"][at] = flat["theta"][at]
    return dict(out, **flat)


def exact(case, seed):
    s = prepare(case, seed)
    family = case["family"]
    return (_exact_xent if family == "xent" else _exact_block if family == "block" else _exact_tensors)(s)
