"""Microscaled 4-bit values (OCP Microscaling MXFP4), and the layer's inference on
expert weights held in them.

Serving a few tokens is bound by reading the experts' weights; in 4 bits, with a scale
byte for each 32 values along the axis that a product sums over, a weight takes 17/32 of
a byte instead of two. ``quantize_experts`` makes the layer's weights ready once;
``forward`` is ``layer.forward`` on them: the same router, index build and combine, the
experts' products by moe_mx_gemm, on bfloat16 rows or (``rows="mx"``) on rows quantised
to 4 bits themselves, which the scaled matrix instructions multiply four times as fast as
bfloat16 ones (3.8 times in loops of either alone; whole products 2.1 to 2.8 times where
an expert has hundreds of rows). Inference only: the weights have no gradient.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B
from . import layer
from .layer import _on


class MX(NamedTuple):
    """Values [..., K]: codes [..., K/2] uint8, value 2i in the low half of byte i, and
    scales [..., K/32] uint8, 2^(s - 127) each."""
    codes: torch.Tensor
    scales: torch.Tensor

    @property
    def shape(self):
        return (*self.codes.shape[:-1], 2 * self.codes.shape[-1])

    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()


class MXExperts(NamedTuple):
    """An expert layer's weights, each [E, N, K] with K the axis summed over."""
    w1: MX             # [E, f, d]
    w3: MX | None      # [E, f, d]; None for a non-gated expert
    w2: MX             # [E, d, f]


def quantize(x, transpose: bool = False, stream=None) -> MX:
    """``x`` [..., R, K] (bfloat16 or float32) in 4 bits, with a scale for each 32 values
    along K; with ``transpose`` of [..., K, R] (R even), whose result is laid out
    [..., R, K]."""
    if stream is not None:
        with _on(stream):
            return quantize(x, transpose)
    shape = x.shape
    if len(shape) < 2:
        raise ValueError("x: %d dimensions, at least 2 needed" % len(shape))
    R, K = shape[-2:]
    if transpose:
        R, K = K, R
    if K % 32:
        raise ValueError("K = %d is not a multiple of 32" % K)
    lead, flags, dev = shape[:-2], B.dtype_flag(x), x.device
    px, = B._args(B._current(), (x, 0, x.dtype, "x"))
    codes = torch.empty((*lead, R, K // 2), dtype=torch.uint8, device=dev)
    scales = torch.empty((*lead, R, K // 32), dtype=torch.uint8, device=dev)
    B._check(B.load_library().moe_mx_quantize(
        px, lead.numel(), R, K, flags | (B.MOE_TRANSPOSED if transpose else 0), codes.data_ptr(),
        scales.data_ptr(), B._stream(None)))
    return MX(codes, scales)


def dequantize(q: MX, dtype=torch.bfloat16, stream=None):
    """The values of ``q`` as bfloat16 or float32 (exact inside the type's range)."""
    if stream is not None:
        with _on(stream):
            return dequantize(q, dtype)
    codes, scales = q
    *lead, half = codes.shape
    K = 2 * half
    if scales.shape != (*lead, K // 32) or K % 32:
        raise ValueError("codes %s and scales %s do not belong together" %
                         (tuple(codes.shape), tuple(scales.shape)))
    u8 = torch.uint8
    pc, ps = B._args(B._current(), (codes, 0, u8, "codes"), (scales, 0, u8, "scales"))
    out = torch.empty((*lead, K), dtype=dtype, device=codes.device)
    if K:
        B._check(B.load_library().moe_mx_dequantize(pc, ps, codes.numel() // half, K, B.dtype_flag(out),
                                                    out.data_ptr(), B._stream(None)))
    return out


ACT = {"none": 0, "silu": B.MOE_ACT_SILU, "relu": B.MOE_ACT_RELU, "swiglu": B.MOE_GATED}


def product(x, w: MX, offsets, rows=None, w3: MX | None = None, act: str = "none", out=None,
            stream=None):
    """out[s] = act(x[rows[s]] w[e]^T) for the slots offsets[e] <= s < offsets[e + 1] of
    each expert e: "none", "silu", "relu", or "swiglu", SiLU(x w^T) * (x w3^T).

    ``x``: bfloat16 [T, K], or MX. ``w``, ``w3``: MX [E, N, K]. ``rows``: int32 [S], the
    row of x of each slot (expert_token_indices); None: slot s is row s. Returns ``out``
    [S, N] bfloat16 (no input's memory); rows at or behind offsets[E] are not written."""
    if stream is not None:
        with _on(stream):
            return product(x, w, offsets, rows, w3, act, out)
    if act not in ACT:
        raise ValueError("act %r is none of %s" % (act, sorted(ACT)))
    if (act == "swiglu") != (w3 is not None):
        raise ValueError("w3 goes with act='swiglu'")
    E, N, K = w.shape
    if w3 is not None and w3.shape != (E, N, K):
        raise ValueError("w3: %s, w is %s" % (tuple(w3.shape), (E, N, K)))
    xc, xs = x if isinstance(x, MX) else (x, None)
    T, Kx = xc.shape
    if xs is not None:
        Kx *= 2
    if Kx != K:
        raise ValueError("x: rows of %d, w sums over %d" % (Kx, K))
    S = T if rows is None else rows.numel()
    if out is None:
        out = torch.empty((S, N), dtype=torch.bfloat16, device=xc.device)
    elif out.shape != (S, N):
        raise ValueError("out: %s, expected %s" % (tuple(out.shape), (S, N)))
    B.moe_mx_gemm(xc, xs, w.codes, w.scales, *(w3 or (None, None)), offsets, rows, T, S, K, N, E,
                  ACT[act], out, None)
    return out


def quantize_experts(w1, w3, w2, stream=None) -> MXExperts:
    """The layer's expert weights (w1, w3 [E, d, f], w2 [E, f, d]; w3 None for a non-gated
    expert) in 4 bits, laid out for ``product``."""
    return MXExperts(quantize(w1, True, stream), None if w3 is None else quantize(w3, True, stream),
                     quantize(w2, True, stream))


def forward(x, w_gate, bias, experts: MXExperts, k: int, renorm: bool, act: str = "swiglu",
            rows: str = "bf16", stream=None):
    """The layer's forward on quantised experts: y [T, d], nothing kept for a backward.
    ``rows``: what the products read beside the weights, "bf16" or "mx" (x and the hidden
    rows quantised to 4 bits, a scale for each 32 values)."""
    if rows not in ("bf16", "mx"):
        raise ValueError("rows %r is neither 'bf16' nor 'mx'" % rows)
    if act not in B.ACT_FLAG:
        raise ValueError("act %r is none of %s" % (act, sorted(B.ACT_FLAG)))
    if x.dtype != torch.bfloat16:
        raise ValueError("x: dtype %s, expected torch.bfloat16" % x.dtype)
    T, d = x.shape
    E, f, K = experts.w1.shape
    if K != d or experts.w2.shape != (E, d, f):
        raise ValueError("experts: %s and %s do not fit rows of %d" %
                         (tuple(experts.w1.shape), tuple(experts.w2.shape), d))
    with _on(stream):
        if T == 0:
            return torch.empty_like(x)
        ids, gates, _ = layer._route(x, w_gate, bias, E, k, renorm, B.MOE_BF16)
        _, offsets, eti, tim, _ = layer._maps(ids, T, E, k)
        xr = quantize(x) if rows == "mx" else x
        h = product(xr, experts.w1, offsets, eti, experts.w3 if act == "swiglu" else None, act)
        O = product(quantize(h) if rows == "mx" else h, experts.w2, offsets)
        y = torch.empty_like(x)
        B.moe_combine(O, gates, tim, T, d, k, B.MOE_BF16, y, None)
    return y
