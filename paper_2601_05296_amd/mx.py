"""Microscaled 4-bit values (OCP Microscaling MXFP4), and the layer's inference on
expert weights held in them.

Serving a few tokens is bound by reading the experts' weights; in 4 bits, with a scale
byte for each 32 values along the axis that a product sums over, a weight takes 17/32 of
a byte instead of two. ``quantize_experts`` makes the layer's weights ready once;
``forward`` is ``layer.forward`` on them: the same router, index build and combine, the
experts' products by moe_mx_gemm, on bfloat16 rows or (``rows="mx"``) on rows quantised
to 4 bits themselves, which the scaled matrix instructions multiply at four times the
bfloat16 rate. Inference only: the weights have no gradient.
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
    along K; with ``transpose`` of [..., K, R], whose result is laid out [..., R, K]."""
    if x.dim() < 2:
        raise ValueError("x: %d dimensions, at least 2 needed" % x.dim())
    R, K = x.shape[-2:]
    if transpose:
        R, K = K, R
    if K % 32:
        raise ValueError("K = %d is not a multiple of 32" % K)
    lead = x.shape[:-2]
    with _on(stream):
        codes = torch.empty((*lead, R, K // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((*lead, R, K // 32), dtype=torch.uint8, device=x.device)
        flags = B.dtype_flag(x) | (B.MOE_TRANSPOSED if transpose else 0)
        B.moe_mx_quantize(x, lead.numel(), R, K, flags, codes, scales, None)
    return MX(codes, scales)


def dequantize(q: MX, dtype=torch.bfloat16, stream=None):
    """The values of ``q`` as bfloat16 or float32 (exact inside the type's range)."""
    K = 2 * q.codes.shape[-1]
    if q.scales.shape != (*q.codes.shape[:-1], K // 32) or K % 32:
        raise ValueError("codes %s and scales %s do not belong together" %
                         (tuple(q.codes.shape), tuple(q.scales.shape)))
    with _on(stream):
        out = torch.empty(q.shape, dtype=dtype, device=q.codes.device)
        B.moe_mx_dequantize(q.codes, q.scales, out.numel() // K if K else 0, K, B.dtype_flag(out),
                            out, None)
    return out


ACT = {"none": 0, "silu": B.MOE_ACT_SILU, "relu": B.MOE_ACT_RELU, "swiglu": B.MOE_GATED}


def product(x, w: MX, offsets, rows=None, w3: MX | None = None, act: str = "none", out=None,
            stream=None):
    """out[s] = act(x[rows[s]] w[e]^T) for the slots offsets[e] <= s < offsets[e + 1] of
    each expert e: "none", "silu", "relu", or "swiglu", SiLU(x w^T) * (x w3^T).

    ``x``: bfloat16 [T, K], or MX. ``w``, ``w3``: MX [E, N, K]. ``rows``: int32 [S], the
    row of x of each slot (expert_token_indices); None: slot s is row s. Returns ``out``
    [S, N] bfloat16; rows at or behind offsets[E] are not written."""
    if act not in ACT:
        raise ValueError("act %r is none of %s" % (act, sorted(ACT)))
    if (act == "swiglu") != (w3 is not None):
        raise ValueError("w3 goes with act='swiglu'")
    E, N, K = w.shape
    if w3 is not None and w3.shape != w.shape:
        raise ValueError("w3: %s, w is %s" % (tuple(w3.shape), tuple(w.shape)))
    xc, xs = x if isinstance(x, MX) else (x, None)
    T, Kx = xc.shape
    if (2 * Kx if xs is not None else Kx) != K:
        raise ValueError("x: rows of %d, w sums over %d" % (2 * Kx if xs is not None else Kx, K))
    S = T if rows is None else rows.numel()
    with _on(stream):
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
