"""The residual update between two blocks of a Peri-LN decoder and its
gradients (``mtdao_peri_norm_*`` of ``include/mtdao.h``), on torch tensors:

    y = residual_scale * x + gate * (post_weight * norm(f) + post_bias)
    h = pre_weight * norm(y) + pre_bias

x is the residual stream, f the output of the block just run; y goes on as the
stream, h is the next block's input.  ``norm``: "rms" or "layer", over the last dimension.
``gate``: None, [d] (a gate per channel), or [G, d] with G a divisor of the number of
rows: consecutive rows share a gate row (G = batch: one a sequence, G = rows: one an
element).  x is fp32 or bf16, f bf16 or fp32 (fp32 only with an fp32 stream);
weights, biases and gate may be either.  ``peri_norm`` is differentiable.
"""
from __future__ import annotations

import torch

import paper_2510_05361_gb300 as P

_CODES = {torch.float32: P.F32, torch.bfloat16: P.BF16}
_NORMS = {"rms": P.NORM_RMS, "layer": P.NORM_LAYER}


def _rows(t, what, d, device):
    """t as [rows, d], sharing its memory."""
    if t.dtype not in _CODES:
        raise ValueError("%s: dtype %s not supported" % (what, t.dtype))
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError("%s must have rows" % what)
        t = t.view(-1, t.shape[-1])           # raises where the rows have no common stride
    if t.shape[1] != d:
        raise ValueError("%s: rows of %d elements, expected %d" % (what, t.shape[1], d))
    if t.device != device or not t.is_cuda:
        raise ValueError("%s must be in device memory, with the others" % what)
    return t


def _stride(t, what):
    if t.shape[0] <= 1:
        if t.shape[1] > 1 and t.numel() and t.stride(1) != 1:
            raise ValueError("%s: rows must be contiguous" % what)
        return t.shape[1]
    if (t.stride(1) != 1 and t.shape[1] > 1) or t.stride(0) < t.shape[1]:
        raise ValueError("%s: rows must be contiguous and apart" % what)
    return t.stride(0)


def _vector(t, what, d, device, like=None):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != d or not t.is_contiguous() or t.device != device:
        raise ValueError("%s must be a contiguous vector of %d elements, with the others" % (what, d))
    if t.dtype not in _CODES or (like is not None and t.dtype != like.dtype):
        raise ValueError("%s: dtype %s not supported, or not that of the other weights" % (what, t.dtype))
    return t.data_ptr()


def _describe(rows, d, norm, stream, branch, post_weight, gate, eps, residual_scale, device):
    """The description's leading fields, and the gate's address."""
    if norm not in _NORMS:
        raise ValueError("norm must be 'rms' or 'layer'")
    gate_rows, gate_code, gate_ptr = 0, 0, None
    if gate is not None:
        if gate.dim() not in (1, 2) or gate.shape[-1] != d or not gate.is_contiguous() or gate.device != device:
            raise ValueError("gate must be contiguous, [%d] or [G, %d], with the others" % (d, d))
        if gate.dtype not in _CODES:
            raise ValueError("gate: dtype %s not supported" % gate.dtype)
        gate_rows = 1 if gate.dim() == 1 else gate.shape[0]
        if gate_rows == 0 or rows % gate_rows:
            raise ValueError("gate: %d rows do not divide %d" % (gate_rows, rows))
        gate_code, gate_ptr = _CODES[gate.dtype], gate.data_ptr()
    return (rows, d, _NORMS[norm], _CODES[stream], _CODES[branch], _CODES[post_weight.dtype], gate_code,
            gate_rows, eps, residual_scale), gate_ptr


def peri_norm_forward(x, f, post_weight, pre_weight, *, post_bias=None, pre_bias=None, gate=None,
                      residual_scale: float = 1.0, eps: float = 1e-5, norm: str = "rms", save: bool = False):
    """(y, h, stats); stats ([2, rows, 2]: of f, of y; mean and reciprocal
    deviation) is None unless ``save``.  y has x's shape and type, h f's."""
    if x.shape != f.shape:
        raise ValueError("x and f differ in shape")
    d, device = x.shape[-1] if x.dim() else 0, x.device
    x2, f2 = _rows(x, "x", d, device), _rows(f, "f", d, device)
    pw, qw = _vector(post_weight, "post_weight", d, device), _vector(pre_weight, "pre_weight", d, device, post_weight)
    pb, qb = _vector(post_bias, "post_bias", d, device, post_weight), _vector(pre_bias, "pre_bias", d, device, post_weight)
    head, gp = _describe(x2.shape[0], d, norm, x.dtype, f.dtype, post_weight, gate, eps, residual_scale, device)
    y, h = torch.empty(x.shape, dtype=x.dtype, device=device), torch.empty(f.shape, dtype=f.dtype, device=device)
    stats = torch.empty((2, x2.shape[0], 2), dtype=torch.float32, device=device) if save else None
    shape = P.mtdao_peri_norm(*head, _stride(x2, "x"), _stride(f2, "f"), d, d, d, d, d, d)
    with torch.cuda.device(device):
        P.mtdao_peri_norm_forward(shape, x2.data_ptr(), f2.data_ptr(), pw, pb, qw, qb, gp, y.data_ptr(), h.data_ptr(),
                                  None if stats is None else stats.data_ptr(),
                                  torch.cuda.current_stream().cuda_stream)
    return y, h, stats


def peri_norm_backward(dh, dy, y, f, stats, post_weight, pre_weight, *, post_bias=None, pre_bias=None, gate=None,
                       residual_scale: float = 1.0, norm: str = "rms"):
    """The gradients, by name: x, f, post_weight, pre_weight and, where they
    were given, post_bias, pre_bias, gate.  dh and dy are those of h and y (dy None: zero); y, f,
    stats as the forward pass had them.  A weight's gradient has its type."""
    d, device = f.shape[-1] if f.dim() else 0, f.device
    dh2, y2, f2 = _rows(dh, "dh", d, device), _rows(y, "y", d, device), _rows(f, "f", d, device)
    dy2 = None if dy is None else _rows(dy, "dy", d, device)
    rows = f2.shape[0]
    if dh2.shape[0] != rows or y2.shape[0] != rows or (dy2 is not None and dy2.shape[0] != rows):
        raise ValueError("dh, dy, y and f differ in shape")
    if dh.dtype != f.dtype or (dy is not None and dy.dtype != y.dtype):
        raise ValueError("dh must have f's dtype, dy that of y")
    if stats.shape != (2, rows, 2) or stats.dtype != torch.float32 or not stats.is_contiguous() or stats.device != device:
        raise ValueError("stats must be what the forward pass gave: [2, %d, 2] fp32" % rows)
    pw, qw = _vector(post_weight, "post_weight", d, device), _vector(pre_weight, "pre_weight", d, device, post_weight)
    pb = _vector(post_bias, "post_bias", d, device, post_weight)
    if (post_bias is None) != (pre_bias is None):
        raise ValueError("post_bias and pre_bias come together")
    _vector(pre_bias, "pre_bias", d, device, post_weight)
    head, gp = _describe(rows, d, norm, y.dtype, f.dtype, post_weight, gate, 0.0, residual_scale, device)
    shape = P.mtdao_peri_norm(*head, d, _stride(f2, "f"), _stride(y2, "y"), d,
                              d if dy2 is None else _stride(dy2, "dy"), _stride(dh2, "dh"), d, d)
    out = {"x": torch.empty(y.shape, dtype=y.dtype, device=device),
           "f": torch.empty(f.shape, dtype=f.dtype, device=device),
           "post_weight": torch.empty_like(post_weight), "pre_weight": torch.empty_like(pre_weight)}
    if post_bias is not None:
        out["post_bias"], out["pre_bias"] = torch.empty_like(post_bias), torch.empty_like(pre_bias)
    if gate is not None:
        out["gate"] = torch.empty_like(gate)
    at = lambda name: out[name].data_ptr() if name in out else None  # noqa: E731
    with torch.cuda.device(device):
        need = P.mtdao_peri_norm_workspace(shape)
        work = torch.empty((need,), dtype=torch.uint8, device=device)
        P.mtdao_peri_norm_backward(shape, dh2.data_ptr(), None if dy2 is None else dy2.data_ptr(), y2.data_ptr(),
                                   f2.data_ptr(), stats.data_ptr(), pw, pb, qw, gp, at("x"), at("f"),
                                   at("post_weight"), at("post_bias"), at("pre_weight"), at("pre_bias"), at("gate"),
                                   work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    return out


def _with_rows(t):
    """t, copied if its rows are not contiguous (autograd hands out expanded gradients)."""
    two = t if t.dim() == 2 else None
    return t if t.is_contiguous() or (two is not None and two.stride(1) == 1 and two.stride(0) >= two.shape[1]) \
        else t.contiguous()


class _PeriNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, post_weight, pre_weight, post_bias, pre_bias, gate, residual_scale, eps, norm):
        y, h, stats = peri_norm_forward(x, f, post_weight, pre_weight, post_bias=post_bias, pre_bias=pre_bias,
                                        gate=gate, residual_scale=residual_scale, eps=eps, norm=norm, save=True)
        ctx.save_for_backward(y, f, stats, post_weight, pre_weight, post_bias, pre_bias, gate)
        ctx.residual_scale, ctx.norm = residual_scale, norm
        ctx.set_materialize_grads(False)
        return y, h

    @staticmethod
    def backward(ctx, dy, dh):
        y, f, stats, post_weight, pre_weight, post_bias, pre_bias, gate = ctx.saved_tensors
        dh = torch.zeros_like(f, memory_format=torch.contiguous_format) if dh is None else _with_rows(dh)
        g = peri_norm_backward(dh, None if dy is None else _with_rows(dy), y, f, stats, post_weight, pre_weight,
                               post_bias=post_bias, pre_bias=pre_bias, gate=gate,
                               residual_scale=ctx.residual_scale, norm=ctx.norm)
        return (g["x"], g["f"], g["post_weight"], g["pre_weight"], g.get("post_bias"), g.get("pre_bias"),
                g.get("gate"), None, None, None)


def peri_norm(x, f, post_weight, pre_weight, *, post_bias=None, pre_bias=None, gate=None,
              residual_scale: float = 1.0, eps: float = 1e-5, norm: str = "rms"):
    """(y, h), differentiable with respect to every tensor."""
    return _PeriNorm.apply(x, f, post_weight, pre_weight, post_bias, pre_bias, gate, residual_scale, eps, norm)
