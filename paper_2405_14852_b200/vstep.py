"""User-facing wrapper: a quantised layer resident on the GPU and its V step.

All computation happens in the CUDA library (``binding``); this class only owns
the device tensors, the workspace and the call order
select -> encode -> dequantise of one step (Algorithm 3, V-step lines and
``dequantize_weights``), and what a layer gives to and takes from the pass that its
update comes from.  ``FeedForward`` is such a pass through three layers.
"""
from __future__ import annotations

import warnings
from typing import Optional

import numpy as np
import torch

from . import binding as B
from .synth import SynthLayer


def _codes_to_torch(codes: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(codes))


class VStepLayer:
    def __init__(self, rows, cols, W, g, scale, codebooks, codes, *, eta=1.0, beam=8, max_k=None, group_dim=8):
        self.rows, self.cols = int(rows), int(cols)
        self.W, self.g, self.scale, self.codebooks, self.codes = W, g, scale, codebooks, codes
        self.eta, self.beam = float(eta), int(beam)
        self.group_dim = int(group_dim)
        self.num_groups = self.rows * (self.cols // self.group_dim)
        self.desc = B.make_layer(self.rows, self.cols, W, g, scale, codebooks, codes, eta=self.eta, beam=self.beam,
                                 group_dim=self.group_dim)
        self._ws = None
        self._one = B.OneLayer()
        if max_k is not None:
            self.reserve(max_k)

    @classmethod
    def from_host(cls, L: SynthLayer, device="cuda", max_k=None) -> "VStepLayer":
        dev = torch.device(device)
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        return cls(L.rows, L.cols, up(L.W), up(L.g), up(L.scale), up(L.codebooks), _codes_to_torch(L.codes).to(dev),
                   eta=L.eta, beam=L.beam, max_k=max_k, group_dim=L.group_dim)

    def reserve(self, k: int) -> torch.Tensor:
        """Workspace large enough for select/encode with this k (grown on demand)."""
        need = B.pvt_workspace_bytes(self.desc, k)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.W.device)
            B.pvt_workspace_init(self._ws)
        return self._ws

    def _with_workspace(self, k: int, call):
        """call(workspace) with the workspace at hand; only a call that finds it too small makes it grow (the library
        checks its size before it enqueues anything)."""
        if self._ws is not None:
            try:
                return call(self._ws)
            except B.PvtError as e:
                if e.code != B.PVT_EWORKSPACE:
                    raise
        return call(self.reserve(k))

    def select(self, k: int, idx_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        if idx_out is None:
            idx_out = torch.empty(k, dtype=torch.int32, device=self.W.device)
        self._with_workspace(k, lambda ws: B.pvt_vstep_select(self.desc, k, idx_out, ws))
        return idx_out

    def select_ste(self, buffer: torch.Tensor, k: int, idx_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Selection while the straight-through buffer takes the step (Appendix E): buffer -= eta * g in place."""
        if idx_out is None:
            idx_out = torch.empty(k, dtype=torch.int32, device=self.W.device)
        self._with_workspace(k, lambda ws: B.pvt_vstep_select_ste(self.desc, buffer, k, idx_out, ws))
        return idx_out

    def sample(self, k: int, rule: int, seed: int, idx_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """A random subspace (B.PVT_SAMPLE_UNIFORM / B.PVT_SAMPLE_PROPORTIONAL) instead of the greedy one."""
        if idx_out is None:
            idx_out = torch.empty(k, dtype=torch.int32, device=self.W.device)
        self._with_workspace(k, lambda ws: B.pvt_vstep_sample(self.desc, k, rule, seed, idx_out, ws))
        return idx_out

    def encode_against(self, buffer: torch.Tensor, idx: torch.Tensor, err_out: Optional[torch.Tensor] = None) -> None:
        """Re-encode the listed groups against buffer / scale (the V step's search with W = buffer, zero step)."""
        k = int(idx.numel())
        desc = B.make_layer(self.rows, self.cols, buffer, self.g, self.scale, self.codebooks, self.codes, eta=0.0,
                            beam=self.beam, group_dim=self.group_dim)
        self._with_workspace(k, lambda ws: B.pvt_vstep_encode(desc, idx, k, err_out, ws))

    def encode(self, idx: torch.Tensor, err_out: Optional[torch.Tensor] = None) -> None:
        k = int(idx.numel())
        self._with_workspace(k, lambda ws: B.pvt_vstep_encode(self.desc, idx, k, err_out, ws))

    def dequant(self, out: Optional[torch.Tensor] = None, dtype=torch.float32) -> torch.Tensor:
        if out is None:
            out = torch.empty(self.rows, self.cols, dtype=dtype, device=self.W.device)
        B.pvt_dequant(self.desc, out)
        return out

    def step(self, k: int, idx_out=None, W_hat=None, err_out=None):
        """One V step followed by the dequantisation that opens the next step."""
        if err_out is None:  # the three calls as one
            if idx_out is None:
                idx_out = torch.empty(k, dtype=torch.int32, device=self.W.device)
            self._with_workspace(k, lambda ws: self._one.step(self.desc, k, idx_out, W_hat, ws))
            return idx_out, W_hat
        idx = self.select(k, idx_out)
        self.encode(idx, err_out)
        return idx, self.dequant(W_hat) if W_hat is not None else None

    def step_trust(self, k_max: int, ratio: float = 0.01):
        """V step whose subspace size follows from the trust ratio (Section 4.3, Appendix J): returns the groups
        in rank order (int32 [k_max]), the number kept (int64 [1]) and float64 [2] = squared norm of the
        dequantised matrix before, squared change kept.  All three stay on the device."""
        need = B.pvt_trust_workspace_bytes(self.desc, k_max)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.W.device)
            B.pvt_workspace_init(self._ws)
        idx = torch.empty(k_max, dtype=torch.int32, device=self.W.device)
        n = torch.empty(1, dtype=torch.int64, device=self.W.device)
        stats = torch.empty(2, dtype=torch.float64, device=self.W.device)
        B.pvt_vstep_trust(self.desc, k_max, ratio, idx, n, stats, self._ws)
        return idx, n, stats

    def quantized(self, fmt: Optional[int] = None, tensor_scale: Optional[torch.Tensor] = None,
                  out: Optional[B.Mx] = None) -> B.Mx:
        """The dequantised weights in 4-bit block floating point: what the forward and backward pass before the next V step
        multiplies by (pvt_mx_product, pvt_mx_grad_input).  fmt is B.PVT_MX_E8M0_32 unless given; with `out`, whose format and
        tensor_scale count, it and tensor_scale need not be given and may not say otherwise.

        B.PVT_MX_E4M3_16 wants a tensor_scale, (dequant().abs().amax() / (6 * 448)).reshape(1) (of zeros any positive one): without one, weights of a deviation
        below 0.01 lose precision and below 0.003 most of them are 0, which is warned of."""
        if (fmt if out is None else out.format) == B.PVT_MX_E4M3_16 and (tensor_scale if out is None else out.tensor_scale) is None:
            warnings.warn("PVT_MX_E4M3_16 without a tensor_scale: blocks whose largest magnitude is below 0.006 become 0",
                          stacklevel=2)
        if out is None:
            out = B.new_mx(self.rows, self.cols, B.PVT_MX_E8M0_32 if fmt is None else fmt, tensor_scale, device=self.codes.device)
        elif fmt is not None and fmt != out.format:
            raise ValueError("out has another format")
        elif tensor_scale is not None and (out.tensor_scale is None or tensor_scale.data_ptr() != out.tensor_scale.data_ptr()):
            raise ValueError("out has another tensor_scale, or none")
        B.pvt_mx_quantize(out, self.dequant())
        return out

    def accumulate_grad(self, dy: torch.Tensor, x: B.Mx, first: bool = False, status: Optional[torch.Tensor] = None) -> None:
        """g += dy^T x (Algorithm 3: the gradient of every batch before the V step); with first g = dy^T x."""
        B.pvt_mx_grad_weight(dy, x, self.g, accumulate=not first, status=status)

    def status(self) -> int:
        return B.pvt_status(self.reserve(1))


def _tensor_scale(top: torch.Tensor) -> torch.Tensor:
    """The tensor scale of PVT_MX_E4M3_16 under which the largest magnitude uses the whole range.  A matrix of zeros has the smallest
    normal number: under a scale of 0 its values are no numbers."""
    return (top / (6.0 * 448.0)).clamp_min(torch.finfo(torch.float32).tiny).reshape(1)


def _version(t: torch.Tensor) -> int:
    """counts what PyTorch writes to a tensor's memory (tensors of inference mode are not counted)"""
    return 0 if t.is_inference() else t._version


class FeedForward:
    """The feed-forward half of a student's block, in the pass between two V steps (Algorithm 3, forward and backward lines; the
    paper's models have it in this form): norm of the residual stream, gated pair, and the layer that leads back.

        total = x + residual,  n = norm(total),  y = (f(n gate^T) * (n up^T)) down^T

    Weights and activations are held in 4 bits (``fmt``), gradients go straight through that.  ``backward`` adds to the g of the
    three layers, which their V steps take, and to the gradients of the norm's weights (float64, as ``pvt_adam_update`` takes
    them).  ``quantize`` again after each step.

    ``x_scale`` and ``h_scale`` are the tensor scales (float32 [1], on the device, read by every pass) of n and of f(a) b under
    PVT_MX_E4M3_16; ``take_scales`` makes or renews them from a batch.  Without them blocks of activations whose largest magnitude is
    below 0.094 lose precision, below 0.006 they become 0, and what is above 2688 is cut off: f(a) b of a deviation of 0.005 is 18 %
    off, with a scale 9 %.  That is warned of, once.

    Gradients of the residual stream, dtotal and dx, are of ``grad_dtype``; those by y, by h and by the pair's products are bfloat16,
    which the tensor cores multiply by."""

    def __init__(self, gate: VStepLayer, up: VStepLayer, down: VStepLayer, weight: torch.Tensor,
                 bias: Optional[torch.Tensor] = None, *, kind: int = B.PVT_NORM_RMS, eps: float = 1e-5,
                 activation: int = B.PVT_ACT_SILU, fmt: int = B.PVT_MX_E8M0_32, x_scale: Optional[torch.Tensor] = None,
                 h_scale: Optional[torch.Tensor] = None, grad_dtype: torch.dtype = torch.bfloat16):
        if (gate.rows, gate.cols) != (up.rows, up.cols) or (gate.rows, gate.cols) != (down.cols, down.rows):
            raise ValueError("gate and up have to be of one shape, down of its transpose")
        if weight.numel() != gate.cols or (bias is not None and bias.numel() != gate.cols):
            raise ValueError("the norm has a weight (and bias) for each input of gate and up")
        for scale in (x_scale, h_scale):
            if scale is not None and (fmt != B.PVT_MX_E4M3_16 or scale.dtype != torch.float32 or scale.numel() != 1):
                raise ValueError("x_scale and h_scale have to be one float32 each, for PVT_MX_E4M3_16")
        if grad_dtype not in (torch.float32, torch.float16, torch.bfloat16):
            raise ValueError("grad_dtype has to be float32, float16 or bfloat16")
        self.x_scale, self.h_scale, self._warned = x_scale, h_scale, False
        self.grad_dtype = grad_dtype
        self.gate, self.up, self.down = gate, up, down
        self.weight, self.bias, self.kind, self.eps, self.activation, self.fmt = weight, bias, kind, eps, activation, fmt
        self.dweight = torch.zeros(gate.cols, dtype=torch.float64, device=weight.device)
        self.dbias = None if bias is None else torch.zeros_like(self.dweight)
        self._status = torch.zeros(1, dtype=torch.int32, device=weight.device)
        self.w_gate = self.w_up = self.w_down = self._scales = self._kept = self._workspace = None

    def quantize(self) -> None:
        """The three layers' weights, as their codes are now, in 4 bits, where they were before: captured passes read the new ones.
        Of PVT_MX_E4M3_16 gate and up share a tensor scale: the gradient by their common input is one sum over both."""
        shared = own = None
        if self.fmt == B.PVT_MX_E4M3_16:
            if self._scales is None:
                self._scales = [torch.empty(1, device=self.weight.device) for _ in range(2)]
            shared, own = self._scales
            top = [layer.dequant().abs().amax() for layer in (self.gate, self.up, self.down)]
            shared.copy_(_tensor_scale(torch.maximum(top[0], top[1])))
            own.copy_(_tensor_scale(top[2]))
        self.w_gate = self.gate.quantized(self.fmt, shared, out=self.w_gate)
        self.w_up = self.up.quantized(self.fmt, shared, out=self.w_up)
        self.w_down = self.down.quantized(self.fmt, own, out=self.w_down)

    def take_scales(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, room: float = 2.0) -> None:
        """x_scale and h_scale of PVT_MX_E4M3_16 from the largest magnitudes of a batch, for others up to ``room`` times as large (what
        is beyond is cut off there).  They are written where they are: captured passes read the new ones."""
        if self.fmt != B.PVT_MX_E4M3_16:
            raise ValueError("tensor scales belong to PVT_MX_E4M3_16")
        if self.w_gate is None:
            self.quantize()
        tokens, device = x.shape[0], x.device
        if self.x_scale is None:
            self.x_scale = torch.empty(1, device=device)
        if self.h_scale is None:
            self.h_scale = torch.empty(1, device=device)
        n, h = (torch.empty(tokens, cols, device=device) for cols in (self.gate.cols, self.gate.rows))
        B.pvt_norm_apply(B.make_norm(x, self.weight, self.bias, kind=self.kind, eps=self.eps, residual=residual), y=n)
        self.x_scale.copy_(_tensor_scale(room * n.abs().amax()))
        xq = B.new_mx(tokens, self.gate.cols, self.fmt, self.x_scale, device=device)
        B.pvt_mx_quantize(xq, n)
        B.pvt_mx_gated(xq, self.w_gate, self.w_up, h=h, activation=self.activation, status=self._status)
        self.h_scale.copy_(_tensor_scale(room * h.abs().amax()))

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None):
        """y (bfloat16) and total (x's type, the next residual) of x [tokens, inputs]; what backward needs is kept until the next call,
        total among it (x itself where there is no residual): it may be written to after backward only, which refuses if PyTorch has
        seen that it was.  (What the calls of ``binding`` write PyTorch does not see.)"""
        if self.w_gate is None:
            self.quantize()
        tokens, device = x.shape[0], x.device
        total = torch.empty_like(x) if residual is not None else x
        stats = torch.empty(tokens, 2, device=device)
        if self.fmt == B.PVT_MX_E4M3_16 and (self.x_scale is None or self.h_scale is None) and not self._warned:
            self._warned = True
            warnings.warn("PVT_MX_E4M3_16 without x_scale or h_scale: blocks of activations whose largest magnitude is below 0.006 become 0",
                          stacklevel=2)
        xq = B.new_mx(tokens, self.gate.cols, self.fmt, self.x_scale, device=device)
        hq = B.new_mx(tokens, self.gate.rows, self.fmt, self.h_scale, device=device)
        y = torch.empty(tokens, self.down.rows, dtype=torch.bfloat16, device=device)
        n = B.make_norm(x, self.weight, self.bias, kind=self.kind, eps=self.eps, residual=residual)
        B.pvt_norm_apply(n, quantized=xq, total=total if residual is not None else None, stats=stats)
        B.pvt_mx_gated(xq, self.w_gate, self.w_up, quantized=hq, activation=self.activation, status=self._status)
        B.pvt_mx_product(hq, self.w_down, y, status=self._status)
        self._kept, self._version = (total, stats, xq, hq), _version(total)
        return y, total

    def backward(self, dy: torch.Tensor, dtotal: Optional[torch.Tensor] = None, first: bool = False) -> torch.Tensor:
        """The gradient by x and by the residual (one and the same, of grad_dtype) from those by y (bfloat16) and, if anything else
        reads it, by total (of grad_dtype), of the last forward pass and at the weights that it had (no quantize in between).  The
        layers' and the norm's gradients are added to; with first they start anew."""
        if self._kept is None:
            raise RuntimeError("backward follows a call of forward")
        total, stats, xq, hq = self._kept
        if _version(total) != self._version:
            raise RuntimeError("x or total has been written to since forward: the gradient would be another's")
        tokens, device = total.shape[0], total.device
        if dtotal is not None:  # (before any gradient has been added to)
            B._matrix(dtotal, tokens, self.gate.cols, "dtotal")
            if dtotal.dtype != self.grad_dtype:
                raise ValueError("dtotal has to be of grad_dtype")
        dh, dup = (torch.empty(tokens, self.gate.rows, dtype=torch.bfloat16, device=device) for _ in range(2))
        dx = torch.empty(tokens, self.gate.cols, dtype=self.grad_dtype, device=device)
        B.pvt_mx_grad_input(dy, self.w_down, dh, status=self._status)
        self.down.accumulate_grad(dy, hq, first=first, status=self._status)
        dgate = dh
        B.pvt_mx_gated_grad(xq, self.w_gate, self.w_up, dh, dgate, dup, activation=self.activation, status=self._status)
        self.gate.accumulate_grad(dgate, xq, first=first, status=self._status)
        self.up.accumulate_grad(dup, xq, first=first, status=self._status)
        B.pvt_mx_gated_grad_input(dgate, dup, self.w_gate, self.w_up, dx, status=self._status)
        n = B.make_norm(total, self.weight, self.bias, kind=self.kind, eps=self.eps)
        if self._workspace is None:  # (of any number of tokens: captured passes write to it)
            self._workspace = B.new_norm_workspace(n, any_rows=True)
        B.pvt_norm_grad(n, stats, dx, dx, dresidual=dtotal, dweight=self.dweight, dbias=self.dbias, accumulate=not first,
                        workspace=self._workspace)
        return dx

    def status(self) -> int:
        """The PVT_DEV_* bits of all passes since the last call, which clears them (it waits for those on the current stream).  Where
        there are any, what these passes wrote is invalid, the gradients that were added to included."""
        bits = int(self._status.item())
        if bits:
            self._status.zero_()
        return bits
