"""Convenience wrappers on torch tensors: one Winograd-aware quantized conv layer (a Plan plus the
device buffers it needs: transformed weights, workspace), and the layers with 4-bit weights and
group scales: linear_w4, experts_w4, and quantize_w4 for their weights.
All arithmetic happens in the CUDA library; torch only owns memory and streams.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np
import torch

from . import binding
from .binding import Plan
from . import _native_torch  # after torch and the library it links against


class WinogradConv:
    def __init__(self, plan: Plan, device="cuda:0"):
        self.plan = plan
        self.device = torch.device(device)
        self.Uq = torch.empty(plan.weight_bytes, dtype=torch.int8, device=self.device)
        self.ws = torch.empty(max(plan.workspace_bytes, 16), dtype=torch.uint8, device=self.device)
        self.bias = None
        # one element, expanded: what an output looks like (empty_like costs half of empty)
        self._y_like = torch.empty(1, dtype=torch.float32 if plan.out_dtype == 1 else torch.int8,
                                   device=self.device).expand(plan.N, plan.H, plan.W, plan.K)

    def load_weights(self, w_q, bias=None, absmax=None) -> None:
        """w_q: int8 [K,3,3,C] (numpy or torch); runs the weight transform."""
        w = torch.as_tensor(np.ascontiguousarray(w_q) if isinstance(w_q, np.ndarray) else w_q)
        w = w.to(self.device, torch.int8).contiguous()
        self.plan.transform_weights(w, self.Uq, absmax)
        self.bias = None if bias is None else torch.as_tensor(bias).to(self.device, torch.float32).contiguous()
        torch.cuda.current_stream().synchronize()  # w may be freed after return

    def empty_output(self) -> torch.Tensor:
        return torch.empty_like(self._y_like, memory_format=torch.contiguous_format)

    def forward(self, x_dev: torch.Tensor, y_dev: torch.Tensor | None = None) -> torch.Tensor:
        """x_dev: int8 [N,H,W,C] on the device."""
        y = _native_torch.forward(self.plan._address, x_dev, self.Uq, self.bias, y_dev, self.ws, self._y_like)
        if type(y) is int:
            raise binding.WinoError(y, "wino_conv_forward")
        if y is None:      # addresses instead of tensors
            y = self.empty_output() if y_dev is None else y_dev
            self.plan.conv_forward(x_dev, self.Uq, self.bias, y, self.ws)
        return y

    def dump(self, stage: int) -> torch.Tensor:
        """One intermediate of the last forward call (WinoError ERR_UNSUPPORTED if that ran as one
        kernel, as small layers do unless the plan's path is forced)."""
        p = self.plan
        t2 = p.t * p.t
        if stage == binding.STAGE_VQ:
            out = torch.empty((t2, p.T, p.C), dtype=torch.int8, device=self.device)
        elif stage == binding.STAGE_MQ:
            out = torch.empty((t2, p.T, p.K), dtype=torch.int8, device=self.device)
        else:
            out = torch.empty((t2, p.T, p.K), dtype=torch.int32, device=self.device)
        p.debug_dump_stage(stage, out, out.numel() * out.element_size())
        return out


def calibrate(make_plan, x_q, w_q, bias, s_x: float, s_w: float, device="cuda:0"):
    """One-shot max-abs calibration of the four inner stage scales on the GPU
    (stand-in for the paper's moving-average range observers, Table 1 caption).

    make_plan(s_V, s_U, s_M, s_Y) -> Plan builds a plan with the given scales.
    Each scale is max|real value of the stage| / 127, rounded once to fp32, taken
    stage by stage on the already-quantized previous stage.  Returns
    (s_V, s_U, s_M, s_Y) as Python floats."""
    dev = torch.device(device)
    x = torch.as_tensor(np.ascontiguousarray(x_q)).to(dev, torch.int8)
    w = torch.as_tensor(np.ascontiguousarray(w_q)).to(dev, torch.int8)
    b = None if bias is None else torch.as_tensor(bias).to(dev, torch.float32)
    f32 = lambda v: float(np.float32(v))
    scale = lambda mx: f32(mx / 127.0) if mx > 0 else 1.0

    def run(s_V, s_U, s_M, s_Y):
        plan = make_plan(s_V, s_U, s_M, s_Y)
        Uq = torch.empty(plan.weight_bytes, dtype=torch.int8, device=dev)
        ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=dev)
        am = torch.zeros(8, dtype=torch.int32, device=dev)
        plan.transform_weights(w, Uq, am[4:])
        plan.calibrate_forward(x, Uq, b, None, ws, am)
        st = plan.last_status()
        if st != 0:
            raise binding.WinoError(st, "calibrate")
        return am.cpu().numpy().view(np.float32)

    enabled = bool(make_plan(1.0, 1.0, 1.0, 1.0).desc.q_M.enabled)
    a = run(1.0, 1.0, 1.0, 1.0)
    s_V = scale(float(a[0]) * f32(s_x))
    s_U = scale(float(a[4]) * f32(s_w))
    a = run(s_V, s_U, 1.0, 1.0)
    s_M = scale(float(a[1]) * (s_U * s_V)) if enabled else 1.0
    a = run(s_V, s_U, s_M, 1.0)
    s_Y = scale(float(a[3]))
    return s_V, s_U, s_M, s_Y


def calibrate_per_channel(make_plan, x_q, w_q, bias, s_x: float, s_w_K, output_per_channel: bool = False,
                          device="cuda:0"):
    """Max-abs calibration with per-output-channel scales (Section 7) on the GPU.

    make_plan(s_V, s_U, s_M, s_Y, out_dtype) -> Plan builds a plan with the given per-layer
    scales and output type; s_w_K are the scales the filters in w_q were quantized with.
    Stage by stage on the already-quantized previous stage: s_V (one scale, from the
    calibration pass), s_U[k] from the weight transform's per-filter statistic, s_M[k] from
    the int32 Hadamard sums (dumped and reduced with torch: plumbing, not the layer's path),
    then the output: one s_Y (a layer inside a network: the next layer sums over these
    channels) or s_Y[k].  Returns (s_V, s_U_K, s_M_K or None, s_Y or s_Y_K)."""
    dev = torch.device(device)
    x = torch.as_tensor(np.ascontiguousarray(x_q)).to(dev, torch.int8)
    w = torch.as_tensor(np.ascontiguousarray(w_q)).to(dev, torch.int8)
    b = None if bias is None else torch.as_tensor(bias).to(dev, torch.float32)
    s_w_K = np.ascontiguousarray(s_w_K, np.float32)
    f32 = lambda v: float(np.float32(v))
    scale = lambda mx: f32(mx / 127.0) if mx > 0 else 1.0
    scales = lambda arr: np.array([scale(float(v)) for v in arr], np.float32)

    def check(plan):
        st = plan.last_status()
        if st != 0:
            raise binding.WinoError(st, "calibrate_per_channel")

    # input side and the transformed filters
    plan = make_plan(1.0, 1.0, 1.0, 1.0, 0)
    K = plan.K
    plan.set_channel_scales(s_w_K, None, None, None)
    Uq = torch.empty(plan.weight_bytes, dtype=torch.int8, device=dev)
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=dev)
    am = torch.zeros(4, dtype=torch.int32, device=dev)
    amK = torch.zeros(K, dtype=torch.int32, device=dev)
    plan.transform_weights_channel_stats(w, Uq, amK)
    plan.calibrate_forward(x, Uq, b, None, ws, am)
    check(plan)
    s_V = scale(float(am.cpu().numpy().view(np.float32)[0]) * f32(s_x))
    u_max = amK.cpu().numpy().view(np.float32).astype(np.float64) * s_w_K.astype(np.float64)
    s_U_K = scales(u_max)
    enabled = bool(plan.desc.q_M.enabled)

    # Hadamard sums under the final V and U scales
    conv = WinogradConv(make_plan(s_V, 1.0, 1.0, 1.0, 0), device=device)
    conv.plan.set_channel_scales(s_w_K, s_U_K, None, None)
    conv.load_weights(w, b)
    conv.plan.debug_run_stages(3, x, conv.Uq, conv.bias, conv.empty_output(), conv.ws)   # staged at any size
    M = conv.dump(binding.STAGE_M_I32)
    check(conv.plan)
    m_max = M.abs().amax(dim=(0, 1)).cpu().numpy().astype(np.float64)
    s_M_K = scales(m_max * (s_U_K.astype(np.float64) * s_V)) if enabled else None

    # the real-valued output under the final inner scales
    conv = WinogradConv(make_plan(s_V, 1.0, 1.0, 1.0, 1), device=device)
    conv.plan.set_channel_scales(s_w_K, s_U_K, s_M_K, None)
    conv.load_weights(w, b)
    y = conv.forward(x)
    check(conv.plan)
    if output_per_channel:
        return s_V, s_U_K, s_M_K, scales(y.abs().amax(dim=(0, 1, 2)).cpu().numpy())
    return s_V, s_U_K, s_M_K, scale(float(y.abs().max()))


# --- layers with 4-bit weights -----------------------------------------------------------
class W4(NamedTuple):
    """A weight matrix [K, C], or a batch of them, as 4-bit codes with one scale per `group` inputs of an
    output.  codes uint8 [..., K/16, C/128, 16, 4, 16] (K and C rounded up; the layout is wino_packed_t's),
    scales bfloat16 or float16 [..., K/16, groups, 16], zeros uint8 like scales, or None (every zero is 8).
    The functions below take any tuple of these six."""
    codes: torch.Tensor
    scales: torch.Tensor
    zeros: Optional[torch.Tensor]
    K: int
    C: int
    group: int


def _w4_result(r, what: str):
    if type(r) is int:
        raise binding.WinoError(r, what)
    return r


def quantize_w4(weight: torch.Tensor, group: int = 128, symmetric: bool = True, scale_dtype=torch.bfloat16,
                values: bool = False):
    """4-bit codes of `weight` ([K, C] or [E, K, C]; float32, bfloat16 or float16, on the GPU), with a scale,
    and unless `symmetric` a zero, for every `group` consecutive inputs (32, 64 or a multiple of 128).  The
    rules are wino_quantize_weights'.  Returns a W4; with values=True also the values that the codes stand
    for, in the weights' type (what quantization-aware training puts in the weights' place).  No gradient goes
    through it: with `v` the values, `weight + (v - weight).detach()` passes one straight through."""
    codes, scales, zeros, K, C, back = _w4_result(
        _native_torch.quantize_w4(weight, group, symmetric, scale_dtype, values), "wino_quantize_weights")
    w = W4(codes, scales, zeros, K, C, group)
    return (w, back) if values else w


def linear_w4(x: torch.Tensor, w, bias: Optional[torch.Tensor] = None, q_x=None, q_Y=None, out_dtype=None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., C] times the transpose of w (W4) plus bias (float32 [K]): [..., K].

    x is float32, bfloat16 or float16, or int8 codes with their quantizer q_x (scale, zero_point), as a
    convolution of this package leaves them.  The result has x's type (float32 for codes), `out_dtype`, or
    with q_Y int8 codes.  out: a tensor to write to, whose rows may be strided, and which may not overlap an input.
    Made for few rows; forward only (inputs and scales that ask for a gradient or carry a forward-mode tangent are
    refused).  Runs on the current stream of x's device."""
    return _w4_result(_native_torch.linear_w4(x, w, bias, q_x, q_Y, out_dtype, out), "wino_linear_forward")


def experts_w4(x: torch.Tensor, router: torch.Tensor, gate, up, down, top_k: int,
               router_bias: Optional[torch.Tensor] = None, normalize: bool = True,
               out: Optional[torch.Tensor] = None):
    """A mixture-of-experts layer for a few tokens x [..., D]: softmax of x router^T + router_bias, the top_k
    largest (ties: lowest index), and the sum over them of weight * down(silu(gate(x)) * up(x)).

    router [E, D] has x's type (float32, bfloat16 or float16); gate and up are W4 batches [E, I, D], down
    [E, D, I].  normalize: weights of a token add up to one.  router_bias float32 [E]: -inf takes an expert
    out.  Returns (y [..., D] of x's type, ids int32 [..., top_k], weights float32 [..., top_k]).  out may not
    overlap an input.  Forward only.  Runs on the current stream of x's device."""
    return _w4_result(_native_torch.experts_w4(x, router, gate, up, down, top_k, router_bias, normalize, out),
                      "wino_experts_forward")


def _by_tiles(v: torch.Tensor, fill) -> torch.Tensor:
    """[..., K, groups] -> [..., K/16, groups, 16]."""
    K, groups = v.shape[-2:]
    v = torch.nn.functional.pad(v, (0, 0, 0, -K % 16), value=fill)
    return v.view(*v.shape[:-2], -1, 16, groups).transpose(-1, -2).contiguous()


def pack_w4(codes: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor] = None, group: int = 128) -> W4:
    """A W4 from codes 0..15 (of any type) [..., K, C], scales (bfloat16 or float16) and zeros
    [..., K, groups], as checkpoints hold them.  A rearrangement with torch, done once."""
    *batch, K, C = codes.shape
    groups = -(-C // group)
    if scales.shape != (*batch, K, groups) or (zeros is not None and zeros.shape != scales.shape):
        raise ValueError(f"scales and zeros must be [..., K, groups]: {(*batch, K, groups)}")
    if scales.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("scales must be bfloat16 or float16")
    for v in (codes, zeros):
        if v is not None and not ((v >= 0) & (v <= 15) & (v == v.to(torch.uint8))).all():
            raise ValueError("codes and zeros must be whole numbers 0..15")
    q = torch.nn.functional.pad(codes.to(torch.uint8), (0, -C % 128, 0, -K % 16))
    tiles_K, tiles_C, n = q.shape[-2] // 16, q.shape[-1] // 128, len(batch)
    q = q.view(*batch, tiles_K, 16, tiles_C, 4, 4, 4, 2)          # a r b i t (e / 2) (e % 2)
    q = q.permute(*range(n), n, n + 2, n + 1, n + 4, n + 3, n + 6, n + 5).reshape(*batch, tiles_K, tiles_C, 16, 4, 16, 2)
    return W4((q[..., 0] | q[..., 1] << 4).contiguous(), _by_tiles(scales, 0.0),
              None if zeros is None else _by_tiles(zeros.to(torch.uint8), 8), K, C, group)


def unpack_w4(w):
    """(codes uint8 [..., K, C], scales [..., K, groups], zeros or None): pack_w4 backwards."""
    codes, scales, zeros, K, C, group = w
    *batch, tiles_K, tiles_C, _, _, _ = codes.shape
    n = len(batch)
    q = torch.stack((codes & 15, codes >> 4), -1).view(*batch, tiles_K, tiles_C, 16, 4, 4, 2, 4)   # a b r t i h e/2
    q = q.permute(*range(n), n, n + 2, n + 1, n + 4, n + 3, n + 6, n + 5).reshape(*batch, tiles_K * 16, tiles_C * 128)

    def rows(v):
        return v.transpose(-1, -2).reshape(*batch, tiles_K * 16, v.shape[-2])[..., :K, :].contiguous()
    return q[..., :K, :C].contiguous(), rows(scales), None if zeros is None else rows(zeros)
