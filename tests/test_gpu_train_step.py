"""A worker's whole training step of a small model: a first norm, Peri-LN blocks of resident-expert
layers, the loss of a linear head, all gradients, and clipped AdamW on every parameter.

fp32 against autograd in 64 bits on the same routes.  The layer's parity is 1e-5 normwise in fp32
(its own tests'); a gradient passes at most two layers, three norms and the loss on its way, each of
which adds as much at most, and a norm's backward may double what it is given once: 1e-4.
"""
import pytest
import torch

from paper_2606_19025_amd.layer import LayerNorm, PeriNormMoELayer
from paper_2606_19025_amd.train import AdamW, LinearCrossEntropy

T, D, E, K, H, V, BLOCKS = 96, 64, 8, 2, 64, 211, 2
RESIDENT = [1, 0, 1, 1, 0, 0, 1, 1]
SCALE, LOGITS, ZC, MAX_NORM, LR = 0.5, 0.7, 1e-3, 0.05, 1e-2
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Model:
    """Masters in fp32 (and working copies in dtype), the operators, and one step of all of them."""

    def __init__(self, dtype, seed=3):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=0.2, mean=0.0: (mean + std * torch.randn(*s, generator=g)).cuda()
        n = sum(RESIDENT)
        self.p = dict(first_w=r(D, mean=1.0), first_b=r(D), head=r(V, D))
        for i in range(BLOCKS):
            self.p.update({f"{i}.router": r(E, D), f"{i}.gate_up": r(n, 2 * H, D), f"{i}.down": r(n, D, H),
                           f"{i}.post_weight": r(D, mean=1.0), f"{i}.post_bias": r(D),
                           f"{i}.gate": r(D, mean=0.5), f"{i}.pre_weight": r(D, mean=1.0),
                           f"{i}.pre_bias": r(D)})
        self.dt = dtype
        matrix = lambda k: k == "head" or k.split(".")[-1] in ("router", "gate_up", "down")
        self.low = {k: v.to(dtype) for k, v in self.p.items() if matrix(k)}
        if dtype is torch.float32:
            self.low = {k: v for k, v in self.p.items() if matrix(k)}  # the masters themselves
        self.first = LayerNorm(T, D, dtype=dtype)
        self.blocks = [PeriNormMoELayer(T, D, E, K, H, RESIDENT, dtype=dtype, gate="channel", scale=SCALE)
                       for _ in range(BLOCKS)]
        self.loss = LinearCrossEntropy(T, D, V, dtype=dtype, scale=LOGITS, z_coef=ZC)
        self.opt = None

    def norms(self, i):
        return {k: self.p[f"{i}.{k}"] for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")}

    def layer(self, i):
        return dict(w_router=self.low[f"{i}.router"], w_gate_up=self.low[f"{i}.gate_up"],
                    w_down=self.low[f"{i}.down"])

    def grads(self):
        out = dict(first_w=self.first.dw, first_b=self.first.db, head=self.loss.dw)
        for i, b in enumerate(self.blocks):
            out.update({f"{i}.router": b.layer.dw_router, f"{i}.gate_up": b.layer.dw_gate_up,
                        f"{i}.down": b.layer.dw_down, f"{i}.post_weight": b.norm.d_post_weight,
                        f"{i}.post_bias": b.norm.d_post_bias, f"{i}.gate": b.norm.d_gate,
                        f"{i}.pre_weight": b.norm.d_pre_weight, f"{i}.pre_bias": b.norm.d_pre_bias})
        return out

    def forward_backward(self, x, labels):
        u, ins = self.first.forward(x, self.p["first_w"], self.p["first_b"]), []
        s = x
        for i, b in enumerate(self.blocks):
            ins.append(u)
            s, u = b.forward(s, u, self.norms(i), **self.layer(i))
        self.loss.forward(u, self.low["head"], labels)
        du, dres = self.loss.backward(u, self.low["head"], labels), None
        for i in reversed(range(BLOCKS)):
            du, dres = self.blocks[i].backward(du, dres, ins[i], self.norms(i), **self.layer(i))
        self.dx = self.first.backward(du, x, self.p["first_w"], dres=dres)

    def step(self, x, labels, t=1):
        self.forward_backward(x, labels)
        if self.opt is None:
            names, g = list(self.p), self.grads()
            low = [self.low.get(k) if self.dt is not torch.float32 else None for k in names]
            self.opt = AdamW([self.p[k] for k in names], [g[k] for k in names], theta_bf16=low,
                             max_norm=MAX_NORM, weight_decay=[0.1 * (self.p[k].dim() > 1) for k in names])
        return self.opt.step(t, LR)


def batch(dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, D, generator=g).to(dtype).cuda()
    labels = torch.randint(0, V, (T,), generator=g)
    labels[torch.rand(T, generator=g) < 0.25] = -1
    return x, labels.int().cuda()


def reference(m, x, labels):
    """(loss, gradients by name, gradient of x) in 64 bits, on the routes that the layers took."""
    p = {k: v.double().requires_grad_() for k, v in m.p.items()}
    X = x.double().requires_grad_()
    norm = lambda v, w, b: (v - v.mean(1, keepdim=True)) * (v.var(1, unbiased=False, keepdim=True) + 1e-5) ** -0.5 * w + b
    local = torch.full((E,), -1, dtype=torch.long)
    local[torch.tensor(RESIDENT) == 1] = torch.arange(sum(RESIDENT))
    local = local.cuda()
    s, u = X, norm(X, p["first_w"], p["first_b"])
    for i, b in enumerate(m.blocks):
        q = lambda k: p[f"{i}.{k}"]
        idx = b.layer.topk_idx.long()
        w = torch.softmax((u @ q("router").T).gather(1, idx), 1)
        f = torch.zeros_like(u)
        for j in range(K):
            e = local[idx[:, j]]
            a = torch.bmm(q("gate_up")[e.clamp(min=0)], u[:, :, None])[:, :, 0]
            h = torch.nn.functional.silu(a[:, :H]) * a[:, H:]
            y = torch.bmm(q("down")[e.clamp(min=0)], h[:, :, None])[:, :, 0]
            f = f + torch.where(e >= 0, w[:, j], 0.0)[:, None] * y
        s = s + SCALE * q("gate") * norm(f, q("post_weight"), q("post_bias"))
        u = norm(s, q("pre_weight"), q("pre_bias"))
    z = LOGITS * u @ p["head"].T
    keep = labels >= 0
    lse = torch.logsumexp(z, 1)
    loss = lse - z.gather(1, labels.long().clamp(min=0)[:, None])[:, 0] + ZC * lse ** 2
    loss = loss[keep].mean()
    loss.backward()
    return loss.item(), {k: v.grad for k, v in p.items()}, X.grad


@pytest.mark.gpu
def test_step_matches_autograd(gpu_lib):
    m = Model(torch.float32)
    x, labels = batch(torch.float32, 1)
    m.forward_backward(x, labels)
    loss, ref, dx = reference(m, x, labels)
    total, n = m.loss.total.tolist()
    assert n == int((labels >= 0).sum()) and abs(total / n - loss) <= 1e-5 * abs(loss)
    for k, g in dict(m.grads(), x=m.dx).items():
        r = dx if k == "x" else ref[k]
        err = ((g.double() - r).norm() / r.norm()).item()
        assert err <= 1e-4, f"{k}: {err:.2e}"
    # the clipped AdamW step on these gradients, in 64 bits: a few fp32 roundings of the update and of
    # the parameter
    before = {k: v.clone() for k, v in m.p.items()}
    grads = {k: v.double() for k, v in m.grads().items()}
    norm = sum(float((v ** 2).sum()) for v in grads.values()) ** 0.5
    n2 = m.step(x, labels)
    assert abs(n2[0].item() - norm) <= 1e-6 * norm and norm > MAX_NORM  # (it clips)
    for k, v in m.p.items():
        g = grads[k] * (MAX_NORM / norm)
        decay = 0.1 * (v.dim() > 1)
        update = LR * (g / (g.abs() + 1e-8) + decay * before[k].double())  # step 1: m / c1 = g, v / c2 = g^2
        want = before[k].double() - update
        # (where |g| is near 1e-8, the quotient turns g's relative error of 1e-6 into as much)
        assert ((v.double() - want).abs() <= 1e-5 * LR + 1e-6 * want.abs()).all(), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps_are_the_eager_ones(gpu_lib, dtype):
    """Steps replayed from a graph, with an eager model's own steps between them."""
    dt = DT[dtype]
    m, e = Model(dt), Model(dt)
    data = [batch(dt, s) for s in range(3)]
    live = [v.clone() for v in data[0]]
    assert torch.equal(m.step(*live), e.step(*data[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step(*live, t=2)
    for i in (1, 2, 0, 1):
        for a, b in zip(live, data[i]):
            a.copy_(b)
        graph.replay()
        e.step(*data[i], t=2)
        torch.cuda.synchronize()
        assert torch.equal(m.loss.total, e.loss.total) and torch.isfinite(m.loss.total).all()
        assert torch.equal(m.opt.norm, e.opt.norm) and torch.equal(m.dx, e.dx)
        for k in m.p:
            assert torch.equal(m.p[k], e.p[k]), k
