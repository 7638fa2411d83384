"""One worker's local step through the resident-expert MoE layer.

``ResidentMoELayer`` owns the device buffers of one layer shape and issues the
C entry points in order (through moe_layer_fwd / moe_layer_bwd, one call each);
it computes nothing itself.

Forward:  moe_route_mask -> moe_dispatch -> moe_grouped_ffn_fwd_sets (resident
          experts [+ shared experts on x, identity dispatch]) -> moe_combine_fwd
Backward: moe_combine_bwd -> moe_grouped_ffn_bwd_sets (resident [+ shared,
          writing dx]) -> moe_dispatch_bwd -> moe_route_bwd (adds the router's dx)
Round boundary: moe_expert_delta over the fp32 master copies.

With ``partitioned=True`` the router is partitioned along with the experts
(the paper's default mode, Sec. 3.3; App. D "Router Efficiency"): it holds
only the resident experts' rows ``w_router[E_r, d]``, every token takes
min(k, E_r) routes, all local, and expert ids are local ids.  The same entry
points run with E := E_r and every expert resident.
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as B


def _check_tensor(name, t, shape, dtype, device, owner):
    """Raise ValueError unless t is a contiguous tensor with this shape, dtype and device."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
            and t.device == device and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor, got {type(t).__name__}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the {owner} on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _check_current(device, owner):
    """Raise ValueError unless device is the current GPU: kernels are launched on the current
    device's stream."""
    if device.type != "cuda":
        raise ValueError(f"the {owner} is on {device}, not on a GPU")
    if torch.cuda.current_device() != device.index:
        raise ValueError(f"the {owner} is on {device}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")


def _on(stream):
    """Context in which torch allocates (and fills) on a call's stream: a buffer that the call makes
    may be memory that the current stream still works on, or reuses when the buffer is dropped."""
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


class ResidentMoELayer:
    def __init__(self, T, d, E, k, H, resident, dtype=torch.bfloat16, n_shared_hidden=0,
                 gate="softmax_topk", inv_tau=1.0, device="cuda", partitioned=False,
                 expert="swiglu", canary=False):
        """canary: fill every output and workspace buffer with NaN (integers:
        -7, workspaces: 0xFF bytes) instead of leaving it uninitialised, so
        that tests see any element the kernels fail to write."""
        self.T, self.d, self.E, self.k, self.H = int(T), int(d), int(E), int(k), int(H)
        res = torch.as_tensor(resident, dtype=torch.uint8).reshape(-1)
        assert res.numel() == self.E
        self.E_r = int(res.sum().item())
        self.E_full = self.E
        self.partitioned = bool(partitioned)
        # expert form: SwiGLU ([Wg; Wu] and [G | U], 2H wide) or the paper's
        # SiLU expert (W1 and A, H wide)
        self.act = B.ACTIVATIONS[expert]
        r1 = 2 if self.act == B.MOE_ACT_SWIGLU else 1
        if self.partitioned:
            if self.E_r == 0:
                raise ValueError("a partitioned router needs at least one resident expert")
            # route over the resident experts only: E := E_r, all resident
            self.E = self.E_r
            self.k = min(self.k, self.E_r)
            res = torch.ones(self.E_r, dtype=torch.uint8)
        self.cap = self.T * min(self.k, self.E_r)
        self.dtype = dtype
        self.dt = B.MOE_BF16 if dtype == torch.bfloat16 else B.MOE_F32
        self.gate = B.GATES[gate] if isinstance(gate, str) else int(gate)
        self.inv_tau = float(inv_tau)
        self.Hs = int(n_shared_hidden)
        self.device = device
        dev = torch.device(device)
        T, d, E, k, H, cap = self.T, self.d, self.E, self.k, self.H, self.cap
        f32, i32, act = torch.float32, torch.int32, dtype
        def e(*s, dt=act):
            if not canary:
                return torch.empty(*s, dtype=dt, device=dev)
            fill = 0xFF if dt == torch.uint8 else -7 if dt == torch.int32 else float("nan")
            return torch.full(s, fill, dtype=dt, device=dev)
        self._alloc = e
        self.resident = res.to(dev)
        # routing
        self.logits = e(T, E, dt=f32)
        self.topk_idx = e(T, k, dt=i32)
        self.topk_w = e(T, k, dt=f32)
        self.topk_local = e(T, k, dt=i32)
        # dispatch
        self.counts = e(max(self.E_r, 1), dt=i32)
        self.offsets = e(self.E_r + 1, dt=i32)
        self.perm = e(max(cap, 1), dt=i32)
        self.inv_perm = e(T, k, dt=i32)
        self.ws_dispatch_bytes = B.moe_dispatch_workspace_size(T, k, self.E_r)
        self.ws_dispatch = e(self.ws_dispatch_bytes, dt=torch.uint8)
        # experts
        rows = max(cap, 1)
        self.xp = e(rows, d)
        self.gu = e(rows, r1 * H)
        self.h = e(rows, H)
        self.yp = e(rows, d)
        self.y = e(T, d)
        # backward
        self.dyp = e(rows, d)
        self.dtopk_w = e(T, k, dt=f32)
        self.dgu = e(rows, r1 * H)
        self.dxp = e(rows, d)
        self.dw_gate_up = e(max(self.E_r, 1), r1 * H, d, dt=f32)
        self.dw_down = e(max(self.E_r, 1), d, H, dt=f32)
        self.dx = e(T, d)
        self.dz = e(T, E, dt=f32)
        self.dw_router = e(E, d, dt=f32)
        self.d_bias = e(E, dt=f32)
        self.ws_route_bytes = B.moe_route_bwd_workspace_size(T, d, E)
        self.ws_route = e(self.ws_route_bytes, dt=torch.uint8)
        self.ws_ffn, self.ws_ffn_bytes = None, 0  # sized on the first backward
        self.ws_fwd, self.ws_fwd_bytes = None, 0  # sized on the first forward
        if self.Hs:
            Hs = self.Hs
            self.s_offsets = torch.tensor([0, T], dtype=i32, device=dev)
            self.s_gu = e(T, r1 * Hs)
            self.s_h = e(T, Hs)
            self.s_y = e(T, d)
            self.s_dgu = e(T, r1 * Hs)
            self.s_dw_gate_up = e(1, r1 * Hs, d, dt=f32)
            self.s_dw_down = e(1, d, Hs, dt=f32)

    def set_resident(self, resident):
        """Switch to another resident set of the same size (a new placement,
        Alg. 1).  The caller migrates the expert weights and optimiser state;
        with a partitioned router it also passes the new router rows."""
        res = torch.as_tensor(resident, dtype=torch.uint8).reshape(-1)
        if res.numel() != self.E_full or int(res.sum().item()) != self.E_r:
            raise ValueError("a new resident set must hold the same number of experts")
        if not self.partitioned:
            self.resident.copy_(res.to(self.resident.device))

    # ------------------------------------------------------------ validation
    def _check(self, name, t, shape, dtype=None):
        """Raise ValueError unless t is a contiguous tensor on this layer's
        device with the given shape and dtype (the layer's own by default)."""
        dtype = self.dtype if dtype is None else dtype
        _check_tensor(name, t, shape, dtype, self.resident.device, "layer")

    def _check_weights(self, x, w_router, w_gate_up, w_down, shared_gate_up, shared_down):
        r1 = 2 if self.act == B.MOE_ACT_SWIGLU else 1
        self._check("x", x, (self.T, self.d))
        self._check("w_router", w_router, (self.E, self.d))
        self._check("w_gate_up", w_gate_up, (self.E_r, r1 * self.H, self.d))
        self._check("w_down", w_down, (self.E_r, self.d, self.H))
        if self.Hs:
            self._check("shared_gate_up", shared_gate_up, (1, r1 * self.Hs, self.d))
            self._check("shared_down", shared_down, (1, self.d, self.Hs))
        elif shared_gate_up is not None or shared_down is not None:
            raise ValueError("shared expert weights given to a layer built without them")

    def _sets(self, x, w_gate_up, w_down, shared_gate_up, shared_down, dy=None):
        """The expert sets of a step: the routed experts [, the shared ones]."""
        sets = [B.ffn_set(self.xp, w_gate_up, w_down, self.offsets, self.cap, self.H, self.E_r,
                          self.gu, self.h, yp=self.yp, dyp=self.dyp, dgu=self.dgu, dxp=self.dxp,
                          dw_gate_up=self.dw_gate_up, dw_down=self.dw_down, activation=self.act)]
        if self.Hs:
            # the shared experts see every token with weight 1: their "dispatched
            # rows" are x, their dyp is dy and their dxp is dx
            sets.append(B.ffn_set(x, shared_gate_up, shared_down, self.s_offsets, self.T, self.Hs,
                                  1, self.s_gu, self.s_h, yp=self.s_y, dyp=dy, dgu=self.s_dgu,
                                  dxp=self.dx, dw_gate_up=self.s_dw_gate_up,
                                  dw_down=self.s_dw_down, activation=self.act))
        return sets

    def _step(self, sets, ws, ws_bytes, x, w_router, router_bias=None, dy=None, accumulate_dw=0):
        """The arguments of moe_layer_fwd / moe_layer_bwd, from this call's tensors and the
        layer's buffers as they are now."""
        p = torch.Tensor.data_ptr
        return B.moe_layer(
            self.dt, self.T, self.d, self.E, self.k, self.E_r, self.gate, accumulate_dw, len(sets),
            self.inv_tau, p(x), p(w_router), None if router_bias is None else p(router_bias),
            p(self.resident), p(self.logits), p(self.topk_idx), p(self.topk_w), p(self.topk_local),
            p(self.counts), p(self.offsets), p(self.perm), p(self.inv_perm), p(self.ws_dispatch),
            self.ws_dispatch_bytes, p(ws) if ws_bytes else None, ws_bytes, p(self.y),
            None if dy is None else p(dy), p(self.dtopk_w), p(self.dz), p(self.dw_router),
            p(self.d_bias), p(self.dx), p(self.ws_route), self.ws_route_bytes,
            (B.moe_ffn_set * 2)(*sets))

    # ------------------------------------------------------------------ forward
    def forward(self, x, w_router, w_gate_up, w_down, router_bias=None, shared_gate_up=None,
                shared_down=None, stream=None, hook=None):
        """hook: called before each library call (e.g. a cache flush between
        kernels for cold per-kernel timing); None in normal use."""
        T, d, E, k, cap, dt = self.T, self.d, self.E, self.k, self.cap, self.dt
        self._check_weights(x, w_router, w_gate_up, w_down, shared_gate_up, shared_down)
        if router_bias is not None:
            self._check("router_bias", router_bias, (E,), torch.float32)
        sets = self._sets(x, w_gate_up, w_down, shared_gate_up, shared_down)
        if self.ws_fwd is None:
            self.ws_fwd_bytes = B.moe_grouped_ffn_fwd_workspace_size(sets, dt, d)
            with _on(stream):
                self.ws_fwd = self._alloc(max(self.ws_fwd_bytes, 1), dt=torch.uint8)
        if hook is None:
            B.moe_layer_fwd(self._step(sets, self.ws_fwd, self.ws_fwd_bytes, x, w_router,
                                       router_bias), stream)
            return self.y
        hook()
        B.moe_route_mask(x, w_router, router_bias, dt, T, d, E, k, self.inv_tau, self.gate,
                         self.resident, self.logits, self.topk_idx, self.topk_w, self.topk_local,
                         stream)
        hook()
        B.moe_dispatch(x, dt, T, d, k, self.E_r, self.topk_local, self.counts, self.offsets,
                       self.perm, self.inv_perm, self.xp, self.ws_dispatch, self.ws_dispatch_bytes,
                       stream)
        hook()
        B.moe_grouped_ffn_fwd_sets(sets, dt, d, self.ws_fwd if self.ws_fwd_bytes else None,
                                   self.ws_fwd_bytes, stream)
        hook()
        B.moe_combine_fwd(self.yp, dt, T, d, k, cap, self.topk_w, self.inv_perm,
                          self.s_y if self.Hs else None, self.y, stream)
        return self.y

    # ----------------------------------------------------------------- backward
    def backward(self, dy, x, w_router, w_gate_up, w_down, shared_gate_up=None, shared_down=None,
                 accumulate_dw=0, stream=None, hook=None):
        T, d, E, k, cap, dt = self.T, self.d, self.E, self.k, self.cap, self.dt
        self._check_weights(x, w_router, w_gate_up, w_down, shared_gate_up, shared_down)
        self._check("dy", dy, (T, d))
        sets = self._sets(x, w_gate_up, w_down, shared_gate_up, shared_down, dy)
        if self.ws_ffn is None:
            self.ws_ffn_bytes = B.moe_grouped_ffn_bwd_workspace_size(sets, dt, d)
            with _on(stream):
                self.ws_ffn = self._alloc(self.ws_ffn_bytes, dt=torch.uint8)
        if hook is None:
            B.moe_layer_bwd(self._step(sets, self.ws_ffn, self.ws_ffn_bytes, x, w_router, dy=dy,
                                       accumulate_dw=accumulate_dw), stream)
            return self.dx
        hook()
        B.moe_combine_bwd(dy, self.yp, dt, T, d, k, cap, self.topk_w, self.inv_perm, self.dyp,
                          self.dtopk_w, stream)
        hook()
        B.moe_grouped_ffn_bwd_sets(sets, dt, d, accumulate_dw, self.ws_ffn, self.ws_ffn_bytes,
                                   stream)
        hook()
        B.moe_dispatch_bwd(self.dxp, dt, T, d, k, cap, self.inv_perm, self.dx, 1 if self.Hs else 0,
                           stream)
        hook()
        B.moe_route_bwd(x, w_router, dt, T, d, E, k, self.inv_tau, self.gate, self.topk_idx,
                        self.topk_w, self.logits, self.dtopk_w, self.dz, self.dw_router,
                        self.d_bias, self.dx, 1, self.ws_route, self.ws_route_bytes, stream)
        return self.dx


class LayerNorm:
    """The layer's pre-norm over [T, d] activations: moe_layernorm_fwd / _bwd on buffers of its
    own (y, mean, rstd, dw, db; dx from the first backward on), which the next call reuses:
    calls on different streams need a norm each.  A call on another stream than the one current
    at construction, where dw and db are set to zero, has to be ordered behind it."""

    def __init__(self, T, d, dtype=torch.bfloat16, bias=True, eps=1e-5, device="cuda"):
        self.T, self.d, self.eps, self.bias = int(T), int(d), float(eps), bool(bias)
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"unsupported dtype {dtype}")
        self.dtype = dtype
        self.dt = B.MOE_BF16 if dtype == torch.bfloat16 else B.MOE_F32
        self.y = torch.empty(self.T, self.d, dtype=dtype, device=device)
        self.mean, self.rstd = (torch.empty(self.T, dtype=torch.float32, device=device)
                                for _ in range(2))
        self.device = self.y.device
        # zeros, and here: the first backward may add to them, in a captured graph too
        self.dw = torch.zeros(self.d, dtype=torch.float32, device=device)
        self.db = torch.zeros_like(self.dw) if self.bias else None
        self.dx = self.ws = None
        self.ws_bytes = 0

    def _check(self, name, t, shape, dtype):
        _check_tensor(name, t, shape, dtype, self.device, "norm")

    def forward(self, x, weight, bias=None, stream=None):
        _check_current(self.device, "norm")
        self._check("x", x, (self.T, self.d), self.dtype)
        self._check("weight", weight, (self.d,), torch.float32)
        if self.bias:
            self._check("bias", bias, (self.d,), torch.float32)
        elif bias is not None:
            raise ValueError("a bias given to a norm built without one")
        B.moe_layernorm_fwd(x, weight, bias, self.dt, self.T, self.d, self.eps, self.y, self.mean,
                            self.rstd, stream)
        return self.y

    def backward(self, dy, x, weight, dres=None, mean=None, rstd=None, accumulate_dw=0,
                 stream=None):
        """dx (+ dres, the residual stream's gradient), with dw and db beside it.  mean and
        rstd: of this x, where they are not those of the last forward."""
        _check_current(self.device, "norm")
        mean = self.mean if mean is None else mean
        rstd = self.rstd if rstd is None else rstd
        for name, t in (("dy", dy), ("x", x)) + ((("dres", dres),) if dres is not None else ()):
            self._check(name, t, (self.T, self.d), self.dtype)
        self._check("weight", weight, (self.d,), torch.float32)
        self._check("mean", mean, (self.T,), torch.float32)
        self._check("rstd", rstd, (self.T,), torch.float32)
        if self.ws is None:
            self.ws_bytes = B.moe_layernorm_bwd_workspace_size(self.T, self.d, self.dt)
            with _on(stream):
                self.dx = torch.empty_like(self.y)
                self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.device)
        B.moe_layernorm_bwd(dy, x, weight, mean, rstd, self.dt, self.T, self.d, dres, self.dx,
                            self.dw, self.db, accumulate_dw, self.ws, self.ws_bytes, stream)
        return self.dx


class PreNormMoELayer:
    """ResidentMoELayer behind its pre-norm, as a transformer block has it: out = x + moe(norm(x)).

    forward returns moe(norm(x)), which the caller adds to x; backward takes the gradient of
    out and returns that of x, the residual's share included.  ``layer`` and ``norm`` hold the
    outputs and gradients of the two."""

    def __init__(self, T, d, E, k, H, resident, dtype=torch.bfloat16, norm_bias=True, eps=1e-5,
                 device="cuda", **kw):
        self.layer = ResidentMoELayer(T, d, E, k, H, resident, dtype=dtype, device=device, **kw)
        self.norm = LayerNorm(T, d, dtype=dtype, bias=norm_bias, eps=eps, device=device)

    def forward(self, x, norm_weight, norm_bias, w_router, w_gate_up, w_down, stream=None, **kw):
        h = self.norm.forward(x, norm_weight, norm_bias, stream=stream)
        return self.layer.forward(h, w_router, w_gate_up, w_down, stream=stream, **kw)

    def backward(self, dout, x, norm_weight, w_router, w_gate_up, w_down, accumulate_dw=0,
                 stream=None, **kw):
        dh = self.layer.backward(dout, self.norm.y, w_router, w_gate_up, w_down,
                                 accumulate_dw=accumulate_dw, stream=stream, **kw)
        return self.norm.backward(dh, x, norm_weight, dres=dout, accumulate_dw=accumulate_dw,
                                  stream=stream)


def _mx_cols(x):
    if not isinstance(x, torch.Tensor) or x.dim() < 2:
        raise ValueError("MXFP4 takes tensors of rows: [..., rows, cols]")
    if x.shape[-1] and x.numel() // x.shape[-1] >= 1 << 31:
        raise ValueError("MXFP4 takes fewer than 2^31 rows")
    return x.shape[-1]


def _one(n_rows):
    """The shape that a tensor of one value has: (1,), or () as it is."""
    return () if isinstance(n_rows, torch.Tensor) and n_rows.dim() == 0 else (1,)


def mxfp4_quantize(x, out=None, n_rows=None, stream=None):
    """(codes, scales) of x [..., rows, cols] in MXFP4: uint8 [..., rows, cols / 2] and
    [..., rows, moe_mxfp4_scale_stride(cols)].  out: such a pair to write to (None: a new one, of
    the call's stream); n_rows: device int32, how many rows to convert (None: all)."""
    cols = _mx_cols(x)
    _check_current(x.device, "tensor")
    rows = x.numel() // cols if cols else 0
    if out is None:
        with _on(stream):
            out = (torch.empty(*x.shape[:-1], cols // 2, dtype=torch.uint8, device=x.device),
                   torch.empty(*x.shape[:-1], B.moe_mxfp4_scale_stride(cols), dtype=torch.uint8,
                               device=x.device))
    codes, scales = out
    _check_tensor("x", x, x.shape, x.dtype, x.device, "tensor")
    _check_tensor("codes", codes, (*x.shape[:-1], cols // 2), torch.uint8, x.device, "tensor")
    _check_tensor("scales", scales, (*x.shape[:-1], B.moe_mxfp4_scale_stride(cols)), torch.uint8,
                  x.device, "tensor")
    if n_rows is not None:
        _check_tensor("n_rows", n_rows, _one(n_rows), torch.int32, x.device, "tensor")
    B.moe_mxfp4_quantize(x, B.dtype_code(x), rows, cols, n_rows, codes, scales, stream)
    return out


def mxfp4_dequantize(codes, scales, dtype=torch.bfloat16, out=None, n_rows=None, stream=None):
    """The values [..., rows, cols] that codes and scales stand for."""
    cols = 2 * _mx_cols(codes)
    _check_current(codes.device, "tensor")
    rows = 2 * codes.numel() // cols if cols else 0
    if out is None:
        with _on(stream):
            out = torch.empty(*codes.shape[:-1], cols, dtype=dtype, device=codes.device)
    _check_tensor("codes", codes, codes.shape, torch.uint8, codes.device, "tensor")
    _check_tensor("scales", scales, (*codes.shape[:-1], B.moe_mxfp4_scale_stride(cols)), torch.uint8,
                  codes.device, "tensor")
    _check_tensor("out", out, (*codes.shape[:-1], cols), dtype, codes.device, "tensor")
    if n_rows is not None:
        _check_tensor("n_rows", n_rows, _one(n_rows), torch.int32, codes.device, "tensor")
    B.moe_mxfp4_dequantize(codes, scales, B.dtype_code(out), rows, cols, n_rows, out, stream)
    return out


class MxFFN:
    """The grouped expert FFN in MXFP4 on up to ``cap`` dispatched rows: moe_mxfp4_quantize of
    the rows, then moe_mxfp4_ffn_fwd on weights given once as (codes, scales) pairs of
    ``mxfp4_quantize``: ``w_gate_up`` of [E_r, 2H (SiLU: H), d], ``w_down`` of [E_r, d, H].
    Its buffers are reused by the next call: calls on different streams need one each.  They are
    made at construction, behind whose stream a call on another one has to be ordered."""

    def __init__(self, cap, w_gate_up, w_down, expert="swiglu"):
        (gu, gu_s), (dn, dn_s) = w_gate_up, w_down
        dev = self.device = gu.device
        r1 = 2 if B.ACTIVATIONS[expert] == B.MOE_ACT_SWIGLU else 1
        self.cap, (E_r, d), H = int(cap), dn.shape[:2], 2 * dn.shape[2]
        self.d, self.H, self.E_r = d, H, E_r
        stride = B.moe_mxfp4_scale_stride
        for name, t, shape in (("w_gate_up codes", gu, (E_r, r1 * H, d // 2)),
                               ("w_gate_up scales", gu_s, (E_r, r1 * H, stride(d))),
                               ("w_down codes", dn, (E_r, d, H // 2)),
                               ("w_down scales", dn_s, (E_r, d, stride(H)))):
            _check_tensor(name, t, shape, torch.uint8, dev, "layer")
        new = lambda *s, dt=torch.uint8: torch.empty(*s, dtype=dt, device=dev)
        self.xq, self.xs = new(self.cap, d // 2), new(self.cap, stride(d))
        self.y = new(self.cap, d, dt=torch.bfloat16)
        ws_bytes = B.moe_mxfp4_ffn_fwd_workspace_size(self.cap, H)
        self.ws = new(max(ws_bytes, 1))
        # (held here: the library keeps addresses only)
        self._held = (gu, gu_s, dn, dn_s)
        p = B._ptr
        self._ffn = B.moe_mxfp4_ffn(
            cap=self.cap, d=d, H=H, n_groups=E_r, activation=B.ACTIVATIONS[expert], x=p(self.xq),
            x_scales=p(self.xs), w_gate_up=p(gu), w_gate_up_scales=p(gu_s), w_down=p(dn),
            w_down_scales=p(dn_s), y=p(self.y), ws=p(self.ws), ws_bytes=ws_bytes)

    def forward(self, xp, offsets, stream=None):
        """y [cap, d] of the dispatched rows xp [cap, d] (bf16 or fp32), whose groups are
        [offsets[g], offsets[g + 1]); rows past offsets[E_r] are neither read nor written."""
        _check_current(self.device, "layer")
        dtype = torch.float32 if getattr(xp, "dtype", None) is torch.float32 else torch.bfloat16
        _check_tensor("xp", xp, (self.cap, self.d), dtype, self.device, "layer")
        _check_tensor("offsets", offsets, (self.E_r + 1,), torch.int32, self.device, "layer")
        B.moe_mxfp4_quantize(xp, B.dtype_code(xp), self.cap, self.d, offsets.data_ptr() + 4 * self.E_r,
                             self.xq, self.xs, stream)
        self._ffn.offsets = offsets.data_ptr()
        B.moe_mxfp4_ffn_fwd(self._ffn, stream)
        return self.y


class InferenceMoELayer:
    """The layer's forward for few tokens on weights that stay: evaluation and generation.

    The weights are given once (they are read where they lie, so later in-place updates are
    seen): ``w_gate_up`` [E_r, 2H, d] and ``w_down`` [E_r, d, H] (SiLU experts: [E_r, H, d]) of
    the router's dtype, or each a (codes, scales) pair of ``mxfp4_quantize``; the shared
    experts' likewise, [1, ...].  ``few`` takes up to 64 tokens; the outputs of its last call
    are y, logits, topk_idx, topk_w and topk_local, in buffers that the next call reuses, whatever
    its number of tokens (two calls on different streams need a layer each)."""

    MAX_TOKENS = 64

    def __init__(self, k, resident, w_router, w_gate_up, w_down, router_bias=None,
                 shared_gate_up=None, shared_down=None, gate="softmax_topk", inv_tau=1.0,
                 expert="swiglu"):
        dev, dt = w_router.device, w_router.dtype
        self.device, self.dtype = dev, dt
        E, d = w_router.shape
        mx = isinstance(w_gate_up, (tuple, list))
        r1 = 2 if B.ACTIVATIONS[expert] == B.MOE_ACT_SWIGLU else 1
        res = torch.as_tensor(resident, dtype=torch.uint8).reshape(-1).to(dev)
        if res.numel() != E:
            raise ValueError(f"resident has {res.numel()} entries, the router {E} experts")
        E_r = int((res != 0).sum().item())

        def inner(w):
            # hidden units of a second projection [n, d, H]
            if isinstance(w, (tuple, list)) != mx:
                raise ValueError("all expert weights are plain, or all are MXFP4 pairs")
            return w[0].shape[-1] * 2 if mx else w.shape[-1]

        H = inner(w_down)
        Hs = inner(shared_down) if shared_down is not None else 0
        if (shared_gate_up is None) != (shared_down is None):
            raise ValueError("shared experts need both shared_gate_up and shared_down")

        def check(name, w, n, rows, cols):
            if isinstance(w, (tuple, list)) != mx:
                raise ValueError(f"{name}: all expert weights are plain, or all are MXFP4 pairs")
            if not mx:
                _check_tensor(name, w, (n, rows, cols), dt, dev, "layer")
                return w, None
            codes, scales = w
            _check_tensor(name + " codes", codes, (n, rows, cols // 2), torch.uint8, dev, "layer")
            _check_tensor(name + " scales", scales, (n, rows, B.moe_mxfp4_scale_stride(cols)),
                          torch.uint8, dev, "layer")
            return codes, scales

        _check_tensor("w_router", w_router, (E, d), dt, dev, "layer")
        if router_bias is not None:
            _check_tensor("router_bias", router_bias, (E,), torch.float32, dev, "layer")
        gu, gu_s = check("w_gate_up", w_gate_up, E_r, r1 * H, d)
        dn, dn_s = check("w_down", w_down, E_r, d, H)
        sgu = sgu_s = sd = sd_s = None
        if Hs:
            sgu, sgu_s = check("shared_gate_up", shared_gate_up, 1, r1 * Hs, d)
            sd, sd_s = check("shared_down", shared_down, 1, d, Hs)
        # (held here: the library keeps addresses only)
        self._held = (w_router, router_bias, res, gu, gu_s, dn, dn_s, sgu, sgu_s, sd, sd_s)
        p = B._ptr
        self.T, self.d, self.E, self.k, self.E_r, self.H, self.Hs = 0, d, E, int(k), E_r, H, Hs
        self._few = B.moe_few(
            dtype=B.dtype_code(w_router), weights=B.MOE_W_MXFP4 if mx else B.MOE_W_PLAIN,
            activation=B.ACTIVATIONS[expert],
            gate=B.GATES[gate] if isinstance(gate, str) else int(gate), d=d, E=E, k=self.k,
            E_r=E_r, H=H, Hs=Hs, inv_tau=float(inv_tau), w_router=p(w_router),
            router_bias=p(router_bias), resident=p(res), w_gate_up=p(gu), w_down=p(dn),
            shared_gate_up=p(sgu), shared_down=p(sd), w_gate_up_scales=p(gu_s),
            w_down_scales=p(dn_s), shared_gate_up_scales=p(sgu_s), shared_down_scales=p(sd_s))
        self.y = self.logits = self.topk_idx = self.topk_w = self.topk_local = self._ws = None

    def _buffers(self):
        """Outputs and workspace for the most tokens that the library takes at this width (the
        workspace grows with them)."""
        f, N = self._few, self.MAX_TOKENS
        new = lambda n, dt: torch.empty(N, n, dtype=dt, device=self.device)
        self._out = dict(y=new(self.d, self.dtype), logits=new(self.E, torch.float32),
                         topk_w=new(self.k, torch.float32), topk_idx=new(self.k, torch.int32),
                         topk_local=new(self.k, torch.int32))
        for name, t in self._out.items():
            setattr(f, name, t.data_ptr())
        for f.T in range(N, 0, -1):
            f.ws_bytes = B.moe_few_fwd_workspace_size(f)
            if f.ws_bytes:  # (0: refused; the call then says what)
                break
        self._ws = torch.empty(max(f.ws_bytes, 1), dtype=torch.uint8, device=self.device)
        f.ws = self._ws.data_ptr()

    def _size(self, T, stream=None):
        """Outputs of T tokens."""
        if not 0 <= T <= self.MAX_TOKENS:
            raise ValueError(f"few takes up to {self.MAX_TOKENS} tokens, got {T}")
        if self._ws is None:
            with _on(stream):
                self._buffers()
        for name, t in self._out.items():
            setattr(self, name, t[:T])
        self.T = self._few.T = T

    def few(self, x, stream=None):
        """y [T, d] of up to 64 tokens x [T, d], by moe_few_fwd."""
        _check_current(self.device, "layer")
        if not isinstance(x, torch.Tensor) or x.dim() != 2:
            raise ValueError("x must be a tensor of tokens: [T, d]")
        if self.y is None or x.shape[0] != self.T:
            self._size(x.shape[0], stream)
        _check_tensor("x", x, (self.T, self.d), self.dtype, self.device, "layer")
        self._few.x = x.data_ptr()
        B.moe_few_fwd(self._few, stream)
        return self.y


def expert_delta(theta_start, theta_now, peers, delta_local=None, delta_avg=None, stream=None):
    """Round-boundary pseudo-gradient of the resident experts and its replica-group average."""
    n = theta_start.numel()
    if delta_avg is None:
        delta_avg = torch.empty_like(theta_start)
    B.moe_expert_delta(theta_start, theta_now, list(peers), len(peers), n, delta_local, delta_avg,
                       stream)
    return delta_avg
