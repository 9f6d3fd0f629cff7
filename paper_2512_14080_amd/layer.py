"""Device buffers for one MoE layer and the call sequence route -> round -> fwd -> bwd (or decode), and for a shared
expert beside it.

Allocation (torch) and argument marshalling only; the work happens in the
library's kernels through the C ABI.
"""
from __future__ import annotations

import numpy as np

from . import binding as B


def _aligned_empty(nbytes: int, device="cuda"):
    import torch
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + nbytes]


def to_device_bf16(bits: np.ndarray, device="cuda"):
    """Raw bf16 bits (uint16 numpy) -> torch.bfloat16 device tensor with the same bits."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    return t.to(device)


def bf16_bits(t) -> np.ndarray:
    """torch bfloat16 tensor -> raw uint16 bits (numpy, host)."""
    import torch
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def bf16_to_f32(t) -> np.ndarray:
    return t.detach().float().cpu().numpy()


def _whole(t, rows, cols):
    """Whether t is contiguous and holds rows of cols elements, under any leading shape ([b,s,cols]) or none."""
    return t.is_contiguous() and t.numel() == rows * cols and (t.dim() == 1 or t.shape[-1] == cols)


def _check_tensor(name, t, dtype, rows, cols, device):
    if t is None or (t.shape == (rows, cols) and t.is_contiguous() and t.dtype == dtype and t.device == device):
        return
    if t.dtype != dtype or t.device != device or not _whole(t, rows, cols):
        raise ValueError(f"{name} must be contiguous {dtype} [{rows}, {cols}] on {device} (got {t.dtype} {list(t.shape)}, "
                         f"strides {t.stride()}, on {t.device})")


def _row_stride(name, t, rows, cols, like):
    """The elements from a row to the next of t, [rows, cols] of like's type and device with whole rows that do not overlap,
    as the dense products take them (0: one after the other)."""
    if t.shape == (rows, cols) and t.is_contiguous() and t.dtype == like.dtype and t.device == like.device:
        return 0
    whole = _whole(t, rows, cols)
    if t.dtype != like.dtype or t.device != like.device or not (whole or t.shape == (rows, cols)):
        raise ValueError(f"{name} must be {like.dtype} [{rows}, {cols}] on {like.device} (got {t.dtype} {list(t.shape)} on "
                         f"{t.device})")
    if whole or (rows == 1 and t.stride(1) == 1):
        return 0
    if t.stride(1) != 1 or not cols <= t.stride(0) < 1 << 30:
        raise ValueError(f"the rows of {name} must be whole and apart (got strides {t.stride()})")
    return t.stride(0)


def _check_device(device, stream):
    if device.type != "cuda":
        raise ValueError(f"the tensors must be on a GPU (they are on {device})")
    import torch
    at = torch.cuda.current_device()
    if at != device.index or (stream is not None and getattr(stream, "device", device) != device):
        raise ValueError(f"the tensors are on {device}, the current device is {at}, the stream {stream}")


class DeviceLayer:
    """All device tensors of one layer invocation.

    ``round_mode`` None runs token-choice routing only; otherwise the layer is
    run on the token-rounded routing with tile ``m_tile``.

    ``held8`` keeps the activations for the backward in 8 bits: "ckpt" with the
    16-bit forward, "quant" with the forward in 8-bit expert products (the
    weights are quantised in every forward, as after an optimiser's step);
    ``keep_x``: X too, and the backward reads that.
    """

    def __init__(self, inputs, round_mode=None, m_tile=None, scores_in=None, u=None, device="cuda",
                 router_grad=True, b1=None, b2=None, keep_logits=True, held8=None, keep_x=False):
        import torch
        if held8 not in (None, "ckpt", "quant"):
            raise ValueError(f'held8 must be None, "ckpt" or "quant" (got {held8!r})')
        if keep_x and held8 is None:
            raise ValueError("keep_x needs held8: the 16-bit layer's backward reads X itself")
        cfg = inputs.cfg
        T, d, n, E, K = inputs.X.shape[0], cfg.d, cfg.n, cfg.E, cfg.K
        self.D = B.dims(T, d, n, E, K)
        self.T, self.d, self.n, self.E, self.K = T, d, n, E, K
        self.X = to_device_bf16(inputs.X, device)
        self.Wr = to_device_bf16(inputs.Wr, device)
        self.W1 = to_device_bf16(inputs.W1, device)
        self.W2 = to_device_bf16(inputs.W2, device)
        self.dO = to_device_bf16(inputs.dO, device)
        self.bias = None if inputs.bias is None else torch.from_numpy(inputs.bias).to(device)
        self.round_mode = round_mode
        self.m_tile = m_tile if m_tile is not None else cfg.m_tile
        flags = (B.MOE_ROUTING_LOGITS if keep_logits else 0) | (B.MOE_ROUTING_SCORES_T if round_mode else 0)
        self.tc = B.Routing(self.D, T * K, flags, device)
        self.tr = None
        if round_mode:
            self.tr = B.Routing(self.D, B.moe_round_capacity(self.D, self.m_tile), 0, device)
        # token rounding builds its own metadata: the token-choice routing
        # only needs its mask, counts and transposed scores
        for_round = (B.MOE_ROUTE_WRITE_SCORES_T | B.MOE_ROUTE_COUNTS_ONLY) if round_mode else 0
        self.route_flags = (B.MOE_ROUTE_WRITE_LOGITS if keep_logits else 0) | for_round
        if scores_in is not None:
            self.tc.arrays()["scores"].copy_(torch.from_numpy(np.ascontiguousarray(scores_in, np.float32)))
            self.route_flags = B.MOE_ROUTE_SCORES_IN | for_round
        self.u = None if u is None else torch.from_numpy(np.asarray(u, np.float32)).to(device)
        cap = self.routing.capacity
        self.held8, self.keep_x = held8, keep_x
        ws_f, ws_b = {None: (B.MOE_WS_FWD, B.MOE_WS_BWD), "ckpt": (B.MOE_WS_FWD_CKPT, B.MOE_WS_BWD_CKPT),
                      "quant": (B.MOE_WS_FWD_QUANT, B.MOE_WS_BWD_CKPT)}[held8]
        self.H = torch.empty((cap, 2 * n), dtype=torch.bfloat16, device=device) if held8 is None else None
        self.ckpt = None if held8 is None else B.Checkpoint(self.D, cap, keep_x, device)
        self.qw = B.QExperts(self.D, device) if held8 == "quant" else None
        self.O = torch.empty((T, d), dtype=torch.bfloat16, device=device)
        self.ws_f = _aligned_empty(B.moe_workspace_bytes(self.D, cap, ws_f), device)
        self.ws_b = _aligned_empty(B.moe_workspace_bytes(self.D, cap, ws_b), device)
        self.dX = torch.empty((T, d), dtype=torch.bfloat16, device=device)
        self.dW1 = torch.empty((E, d, 2 * n), dtype=torch.bfloat16, device=device)
        self.dW2 = torch.empty((E, n, d), dtype=torch.bfloat16, device=device)
        self.router_grad = router_grad
        self.dWr = torch.empty((d, E), dtype=torch.float32, device=device) if router_grad else None
        self.dbias = torch.empty((E,), dtype=torch.float32, device=device) if router_grad else None
        self.dS = torch.empty((cap,), dtype=torch.float32, device=device)
        # optional expert biases (fp32 [E,2n] and [E,d]) and their gradients
        f32 = torch.float32
        self.b1 = None if b1 is None else torch.from_numpy(np.ascontiguousarray(b1, np.float32)).to(device)
        self.b2 = None if b2 is None else torch.from_numpy(np.ascontiguousarray(b2, np.float32)).to(device)
        self.db1 = torch.empty((E, 2 * n), dtype=f32, device=device) if b1 is not None else None
        self.db2 = torch.empty((E, d), dtype=f32, device=device) if b2 is not None else None
        self.eb = B.expert_bias(self.b1, self.b2, self.db1, self.db2)
        # of decode (made here: memory taken in a call belongs to the current stream, not to the call's)
        self.ws_d = None
        if not self.round_mode and scores_in is None:
            which = B.MOE_WS_DECODE if self.qw is None else B.MOE_WS_DECODE_QUANT
            self.ws_d = _aligned_empty(B.moe_workspace_bytes(self.D, T * K, which), device)

    @property
    def routing(self):
        return self.tr if self.round_mode else self.tc

    def route(self, stream=None):
        B.moe_route(self.D, self.X, self.Wr, self.bias, self.route_flags, self.tc, stream)
        if self.round_mode:
            B.moe_round_tokens(self.D, self.m_tile, self.round_mode, self.u, self.tc, self.tr, stream)

    def forward(self, stream=None):
        if self.held8 == "ckpt":
            B.moe_fwd_ckpt(self.D, self.X, self.W1, self.W2, self.routing, self.ckpt, self.O, self.ws_f, stream,
                           eb=self.eb)
            return
        if self.held8 == "quant":
            B.moe_quantize_experts(self.D, self.W1, self.W2, self.qw, stream)
            B.moe_fwd_quant(self.D, self.X, self.qw, self.routing, self.ckpt, self.O, self.ws_f, stream, eb=self.eb)
            return
        B.moe_fwd(self.D, self.X, self.W1, self.W2, self.routing, self.H, self.O, self.ws_f, stream, eb=self.eb)

    def backward(self, stream=None):
        if self.held8:
            B.moe_bwd_ckpt(self.D, self.dO, None if self.keep_x else self.X, self.ckpt, self.W1, self.W2,
                           self.Wr if self.router_grad else None, self.routing, self.dX, self.dW1, self.dW2, self.dWr,
                           self.dbias, self.dS, self.ws_b, stream, eb=self.eb)
            return
        B.moe_bwd(self.D, self.dO, self.X, self.H, self.W1, self.W2, self.Wr if self.router_grad else None,
                  self.routing, self.dX, self.dW1, self.dW2, self.dWr, self.dbias, self.dS, self.ws_b, stream,
                  eb=self.eb)

    def step(self, stream=None):
        self.route(stream)
        self.forward(stream)
        self.backward(stream)

    def rows(self) -> int:
        """P, the number of routed rows (reads the device offsets)."""
        return int(self.routing.arrays()["offsets"][-1].item())

    def decode(self, R=None, stream=None, topk_idx=None, topk_w=None):
        """The forward of a few tokens (T <= MOE_DECODE_MAX_T) in one call, routing included: O = R + the layer's output.
        R is bf16 [T,d]; topk_idx (int32) and topk_w (fp32), [T,K], take the selection.
        Token choice only, on the 8-bit weights with held8="quant" (quantise them first: quantize_experts), where route
        and forward on weights that are quantised already are mostly as fast or faster from two tokens on (moe_decode_quant
        in the header).  Calls share the layer's buffers and must be ordered."""
        if self.round_mode:
            raise ValueError("decode routes by token choice: round_mode must be None")
        if self.route_flags & B.MOE_ROUTE_SCORES_IN:
            raise ValueError("decode routes by softmax(X Wr + bias): scores_in must be None")
        import torch
        device = self.X.device
        _check_tensor("R", R, torch.bfloat16, self.T, self.d, device)
        _check_tensor("topk_idx", topk_idx, torch.int32, self.T, self.K, device)
        _check_tensor("topk_w", topk_w, torch.float32, self.T, self.K, device)
        _check_device(device, stream)
        if self.qw is not None:
            B.moe_decode_quant(self.D, self.X, self.Wr, self.bias, self.qw, R, self.O, self.ws_d, topk_idx, topk_w,
                               stream, eb=self.eb)
        else:
            B.moe_decode(self.D, self.X, self.Wr, self.bias, self.W1, self.W2, R, self.O, self.ws_d, topk_idx, topk_w,
                         stream, eb=self.eb)

    def quantize_experts(self, stream=None):
        if self.qw is None:
            raise ValueError('quantize_experts needs held8="quant"')
        B.moe_quantize_experts(self.D, self.W1, self.W2, self.qw, stream)


class SharedExpert:
    """A dense SwiGLU expert that every token passes through, beside the routed ones:
    Y = R + (SiLU(X Wu_gate) * X Wu_up) Wd, with Wu [d,2m] (gate columns first) and Wd [m,d] in bf16 and optional fp32
    biases [2m] and [d].  ``train`` keeps what the backward reads.

    X, Y, R and the gradients are bf16 [T,d] of exactly T rows (contiguous ones under any leading shape); rows may be further apart than they are long (by a
    multiple of 8 elements), and what lies between them is neither read nor written.  Calls share the object's buffers and
    must be ordered; backward is that of the forward before it."""

    def __init__(self, T, Wu, Wd, bu=None, bd=None, train=False):
        import torch
        d, m = Wu.shape[0], Wd.shape[0]
        if Wu.shape != (d, 2 * m) or Wd.shape != (m, d):
            raise ValueError(f"Wu must be [d, 2m] and Wd [m, d] (got {tuple(Wu.shape)}, {tuple(Wd.shape)})")
        if not (Wu.is_contiguous() and Wd.is_contiguous()):
            raise ValueError("Wu and Wd must be contiguous")
        if Wu.dtype != torch.bfloat16 or Wd.dtype != torch.bfloat16 or Wd.device != Wu.device:
            raise ValueError(f"Wu and Wd must be bfloat16 on one device (got {Wu.dtype} on {Wu.device}, {Wd.dtype} on {Wd.device})")
        for name, b, size in (("bu", bu, 2 * m), ("bd", bd, d)):
            _check_tensor(name, b, torch.float32, 1, size, Wu.device)
        self.T, self.d, self.m, self._sizes = T, d, m, {}
        self.Wu, self.Wd, self.bu, self.bd = Wu, Wd, bu, bd
        dev, bf16, f32 = Wu.device, torch.bfloat16, torch.float32

        def workspace(which):
            # (of any stride: rows that pass 32-bit offsets go another way, whose workspace may be the larger)
            forms = (self._up(0), self._up((1 << 30) - 8), self._down(0, 0))
            return _aligned_empty(max(B.moe_linear_workspace_bytes(L, which) for L in forms), dev)

        def like(t):
            return None if t is None else torch.empty_like(t)

        self.A = torch.empty((T, m), dtype=bf16, device=dev)
        self.ws_f = workspace(B.MOE_WS_LINEAR_FWD)
        self.H = None
        if train:
            self.H = torch.empty((T, 2 * m), dtype=bf16, device=dev)
            self.dA, self.ws_b = torch.empty_like(self.A), workspace(B.MOE_WS_LINEAR_BWD)
            self.dWu, self.dWd, self.dbu, self.dbd = like(Wu), like(Wd), like(bu), like(bd)

    # (the sizes of the two products for given strides, formed once)
    def _up(self, ldx):
        L = self._sizes.get(ldx)
        if L is None:
            L = self._sizes[ldx] = B.linear_dims(self.T, self.d, self.m, "swiglu", ldx=ldx)
        return L

    def _down(self, ldr, ldy):
        L = self._sizes.get((ldr, ldy))
        if L is None:
            L = self._sizes[ldr, ldy] = B.linear_dims(self.T, self.m, self.d, ldr=ldr, ldy=ldy)
        return L

    def _stride(self, name, t):
        return 0 if t is None else _row_stride(name, t, self.T, self.d, self.Wu)

    def forward(self, X, Y, R=None, stream=None):
        up, down = self._up(self._stride("X", X)), self._down(self._stride("R", R), self._stride("Y", Y))
        _check_device(self.Wu.device, stream)
        B.moe_linear_fwd(up, X, self.Wu, self.bu, None, self.H, self.A, self.ws_f, stream)
        B.moe_linear_fwd(down, self.A, self.Wd, self.bd, R, None, Y, self.ws_f, stream)

    def backward(self, dY, X, dX, G=None, stream=None):
        """dX = the gradient through this expert + G (which may be dX itself), and dWu, dWd, dbu, dbd.  X, dX and G have
        their rows equally far apart."""
        if self.H is None:
            raise ValueError("backward needs train=True")
        down, ldx = self._down(0, self._stride("dY", dY)), self._stride("X", X)
        for name, t in (("dX", dX), ("G", G)):
            if t is not None and self._stride(name, t) != ldx:
                raise ValueError(f"the rows of X and {name} must be equally far apart (got {X.stride()}, {t.stride()})")
        _check_device(self.Wu.device, stream)
        B.moe_linear_bwd(down, dY, self.A, self.Wd, None, None, self.dA, self.dWd, self.dbd, self.ws_b, stream)
        B.moe_linear_bwd(self._up(ldx), self.dA, X, self.Wu, self.H, G, dX, self.dWu, self.dbu, self.ws_b, stream)
