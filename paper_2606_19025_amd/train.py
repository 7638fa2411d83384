"""What a worker's training step needs behind its layers: the loss, the gradients' norm, clipping and
AdamW over all parameters.

As in ``layer``, the classes own buffers and issue the C entry points; they compute nothing
themselves.
"""
from __future__ import annotations

import torch

from . import binding as B
from .layer import _check_current, _check_tensor, _on


def _device(tensors, owner):
    """The device of a list of tensors, all contiguous and on it."""
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{owner} {i} must be a tensor, got {type(t).__name__}")
    if not tensors:
        raise ValueError(f"no {owner} given")
    return tensors[0].device


def _disjoint(name, tensors):
    """Raise ValueError if two of the tensors share memory."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), i)
                   for i, t in enumerate(tensors) if t is not None and t.numel())
    for (_, end, i), (begin, _, j) in zip(spans, spans[1:]):
        if begin < end:
            raise ValueError(f"{name} {i} and {j} overlap")


def _apart(name, written, read):
    """Raise ValueError if a written tensor shares memory with one that is read, but for the pair i, i
    where both are the same."""
    spans = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), kind, i)
             for kind, lst in ((0, written), (1, read)) for i, t in enumerate(lst)
             if t is not None and t.numel()]
    ends = [(0, -1), (0, -1)]  # the furthest end so far of each kind, and whose
    for begin, end, kind, i in sorted(spans):
        far, j = ends[1 - kind]
        if begin < far and not (i == j and written[i].data_ptr() == read[i].data_ptr()):
            raise ValueError(f"{name} {i if kind == 0 else j} overlaps an input")
        ends[kind] = max(ends[kind], (end, i))


class LinearCrossEntropy:
    """Softmax cross entropy of N tokens x [N, d] against a vocabulary w [V, d], without the logits
    being kept: moe_xent_fwd, moe_xent_bwd.

    Logits are scale x w^T; z_coef adds z_coef lse^2 to a token's loss.  Labels are int32; a negative
    one leaves its token out.  forward returns ``loss`` [N]; ``lse`` [N] and ``total`` (the sum of the
    losses and the number of tokens that count) stand beside it.  backward, from the last forward's
    lse, returns ``dx`` with ``dw`` beside it, fp32 or of the weights' type (dw_dtype).  The buffers
    are the object's own and are reused by the next call: calls on different streams need one each,
    and a call on another stream than the one current at construction has to be ordered behind it.
    dx, dw and the workspaces are made by the first call that needs them, dw as zeros where that call
    adds to it; one that is captured may not be the first and add."""

    def __init__(self, N, d, V, dtype=torch.bfloat16, scale=1.0, z_coef=0.0, dw_dtype=torch.float32,
                 device="cuda"):
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"unsupported dtype {dtype}")
        if dw_dtype not in (torch.float32, dtype):
            raise ValueError(f"dw_dtype {dw_dtype} is neither float32 nor {dtype}")
        self.N, self.d, self.V, self.dtype, self.dw_dtype = int(N), int(d), int(V), dtype, dw_dtype
        code = lambda t: B.MOE_BF16 if t == torch.bfloat16 else B.MOE_F32
        self.loss, self.lse = (torch.empty(self.N, dtype=torch.float32, device=device) for _ in range(2))
        self.total = torch.empty(2, dtype=torch.float32, device=device)
        self.device = self.total.device
        self.dx = self.dw = self.ws_fwd = self.ws_bwd = None
        self._args = B.moe_xent(
            dtype=code(dtype), N=self.N, d=self.d, V=self.V, scale=float(scale), z_coef=float(z_coef),
            loss=self.loss.data_ptr(), lse=self.lse.data_ptr(), total=self.total.data_ptr(),
            dw_dtype=code(dw_dtype))

    def _inputs(self, x, w, labels):
        _check_current(self.device, "loss")
        for name, t, shape, dtype in (("x", x, (self.N, self.d), self.dtype),
                                      ("w", w, (self.V, self.d), self.dtype),
                                      ("labels", labels, (self.N,), torch.int32)):
            _check_tensor(name, t, shape, dtype, self.device, "loss")
        a = self._args
        a.x, a.w, a.labels = x.data_ptr(), w.data_ptr(), labels.data_ptr()
        return a

    def _workspace(self, size, a):
        n = size(a)
        return torch.empty(max(n, 1), dtype=torch.uint8, device=self.device), n

    def forward(self, x, w, labels, stream=None):
        a = self._inputs(x, w, labels)
        if self.ws_fwd is None:
            with _on(stream):
                self.ws_fwd, self.ws_fwd_bytes = self._workspace(B.moe_xent_fwd_workspace_size, a)
        a.ws, a.ws_bytes = self.ws_fwd.data_ptr(), self.ws_fwd_bytes
        B.moe_xent_fwd(a, stream)
        return self.loss

    def backward(self, x, w, labels, dloss=None, accumulate_dw=0, stream=None):
        """dloss: the losses' gradients [N] fp32, None: of the mean over the tokens that count."""
        a = self._inputs(x, w, labels)
        if dloss is not None:
            _check_tensor("dloss", dloss, (self.N,), torch.float32, self.device, "loss")
        if self.ws_bwd is None:
            with _on(stream):
                ws, n = self._workspace(B.moe_xent_bwd_workspace_size, a)
                dx = torch.empty(self.N, self.d, dtype=self.dtype, device=self.device)
                if accumulate_dw and torch.cuda.is_current_stream_capturing():
                    # (the graph would set dw to zero again at each replay)
                    raise ValueError("a captured backward adds to a dw that an earlier call has made")
                make = torch.zeros if accumulate_dw else torch.empty
                dw = make(self.V, self.d, dtype=self.dw_dtype, device=self.device)
            # (all of them or none: a call without memory for one leaves the object as it was)
            self.dx, self.dw, self.ws_bwd, self.ws_bwd_bytes = dx, dw, ws, n
            a.dx, a.dw = dx.data_ptr(), dw.data_ptr()
        a.dloss, a.accumulate_dw = B._ptr(dloss), int(accumulate_dw)
        a.ws, a.ws_bytes = self.ws_bwd.data_ptr(), self.ws_bwd_bytes
        B.moe_xent_bwd(a, stream)
        return self.dx


class _GradNorm:
    """The norm of the given gradients together, and the scale that limits it: moe_grad_norm.  One that
    is given twice counts twice.  out: where a clipper writes (None: nowhere)."""

    def __init__(self, grads, max_norm, out=None):
        grads = list(grads)
        self.device = _device(grads, "gradient")
        self.max_norm = float(max_norm)
        if not self.max_norm > 0:
            raise ValueError(f"max_norm must be positive, got {max_norm}")
        if out is not None and len(out) != len(grads):
            raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
        for i, g in enumerate(grads):
            if g.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError(f"gradient {i} has dtype {g.dtype}: float32 or bfloat16")
            _check_tensor(f"gradient {i}", g, g.shape, g.dtype, self.device, "clipper")
            if out is not None:
                _check_tensor(f"output {i}", out[i], g.shape, g.dtype, self.device, "clipper")
        self._held = grads, out  # (the library keeps addresses only)
        self.n = len(grads)
        self._grads = (B.moe_grad * self.n)(*[
            B.moe_grad(g.data_ptr(), B._ptr(out and out[i]), g.numel(), B.dtype_code(g))
            for i, g in enumerate(grads)])
        self.ws_bytes = B.moe_grad_norm_workspace_size(self._grads, self.n)
        self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.device)
        self.norm = torch.empty(2, dtype=torch.float32, device=self.device)

    def measure(self, stream=None):
        """[norm, scale] of the gradients as they are."""
        _check_current(self.device, "clipper")
        B.moe_grad_norm(self._grads, self.n, self.max_norm, self.norm, self.ws, self.ws_bytes, stream)
        return self.norm


class GradClipper(_GradNorm):
    """The norm of the given gradients together, and clipping by it: moe_grad_norm, moe_grad_clip.

    grads: contiguous fp32 or bf16 tensors, read where they lie at every call (a layer's gradient
    buffers).  max_norm: infinite measures alone.  out: where the clipped gradients go, tensors like
    grads (None: in place), none of which may overlap another or another's gradient.  ``norm`` holds the
    norm and the scale min(1, max_norm / norm) of the last call, on the GPU; a norm that is not finite
    has the scale NaN and clips nothing.  The workspace is the object's own: calls on different streams
    need one each, and a call on another stream than the one current at construction has to be ordered
    behind it."""

    def __init__(self, grads, max_norm, out=None):
        grads = list(grads)
        out = grads if out is None else list(out)
        super().__init__(grads, max_norm, out)
        _disjoint("outputs", out)
        _apart("output", out, grads)

    def clip(self, stream=None):
        """[norm, scale], and the gradients clipped."""
        self.measure(stream)
        B.moe_grad_clip(self._grads, self.n, self.norm, stream)
        return self.norm


class AdamW:
    """AdamW on many fp32 tensors at once, moe_adamw_steps, with the gradients clipped on the way
    (max_norm; None: as they are).

    theta, m, v: lists of fp32 tensors, updated in place; grads: fp32 or bf16, read where they lie
    at every step (one that is given to several parameters counts as often in the norm); theta_bf16:
    a list of bf16 tensors (or of None among them) that receive the updated parameters.  All are
    16-byte aligned (``GradClipper`` takes gradients as they lie).  weight_decay and lr_scale: a
    number, or one for each tensor.  ``norm`` holds the last step's [norm, scale]; a step whose norm
    is not finite changes nothing.  A step on another stream than the one current at construction,
    where m and v are set to zero, has to be ordered behind it."""

    def __init__(self, theta, grads, m=None, v=None, theta_bf16=None, max_norm=None,
                 betas=(0.9, 0.95), eps=1e-8, weight_decay=0.0, lr_scale=1.0):
        theta, grads = list(theta), list(grads)
        dev = self.device = _device(theta, "parameter")
        n = self.n = len(theta)
        self.m = [torch.zeros_like(t) for t in theta] if m is None else list(m)
        self.v = [torch.zeros_like(t) for t in theta] if v is None else list(v)
        low = [None] * n if theta_bf16 is None else list(theta_bf16)
        each = lambda x: [float(x)] * n if isinstance(x, (int, float)) else [float(y) for y in x]
        decay, rate = each(weight_decay), each(lr_scale)
        for name, lst in (("grads", grads), ("m", self.m), ("v", self.v), ("theta_bf16", low),
                          ("weight_decay", decay), ("lr_scale", rate)):
            if len(lst) != n:
                raise ValueError(f"{len(lst)} {name} for {n} parameters")
        for i, t in enumerate(theta):
            for name, u in (("parameter", t), ("m", self.m[i]), ("v", self.v[i])):
                _check_tensor(f"{name} {i}", u, t.shape, torch.float32, dev, "optimiser")
            g = grads[i]
            if getattr(g, "dtype", None) is not torch.bfloat16:
                _check_tensor(f"gradient {i}", g, t.shape, torch.float32, dev, "optimiser")
            else:
                _check_tensor(f"gradient {i}", g, t.shape, torch.bfloat16, dev, "optimiser")
            if low[i] is not None:
                _check_tensor(f"theta_bf16 {i}", low[i], t.shape, torch.bfloat16, dev, "optimiser")
            for name, u in (("parameter", t), ("gradient", g), ("m", self.m[i]), ("v", self.v[i]),
                            ("theta_bf16", low[i])):
                if u is not None and u.data_ptr() % 16:
                    raise ValueError(f"{name} {i} must be 16-byte aligned")
        _disjoint("tensors", theta + self.m + self.v + low)
        _apart("tensor", theta + self.m + self.v + low, [None] * (4 * n) + grads)
        self.betas, self.eps = (float(betas[0]), float(betas[1])), float(eps)
        self._measured = None if max_norm is None else _GradNorm(grads, max_norm)
        self.norm = None if max_norm is None else self._measured.norm
        self._held = theta, grads, low  # (the library keeps addresses only)
        p = B._ptr
        self._tensors = (B.moe_adamw_tensor * n)(*[
            B.moe_adamw_tensor(p(theta[i]), p(grads[i]), p(self.m[i]), p(self.v[i]), p(low[i]),
                               theta[i].numel(), B.dtype_code(grads[i]), rate[i], decay[i])
            for i in range(n)])

    def step(self, t, lr, stream=None):
        """Step t (1 for the first) at rate lr; returns [norm, scale] (None without max_norm)."""
        _check_current(self.device, "optimiser")
        if self._measured is not None:
            self._measured.measure(stream)
        B.moe_adamw_steps(self._tensors, self.n, int(t), float(lr), *self.betas, self.eps, self.norm,
                          stream)
        return self.norm
