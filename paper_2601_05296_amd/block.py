"""Residual blocks around the MoE layer: norms before and after it, a gate, a residual
scale, forward and backward, and inference on 4-bit experts.

One block, x its residual stream (p = post_norm(y) * w_post, or y without a post-norm):
  n = rms_norm(x) * w_pre;  y = layer(n);  x' = res_scale * x + gate * p
``norm_forward`` does a block's last line and the next block's first in one pass;
``forward`` and ``backward`` chain a list of blocks with it, ``infer`` serves the same
blocks with their experts in 4 bits (mx.py). Rows of the norms: d a multiple of 8, at most
8192, which is a block's limit where the layer has none.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import NamedTuple

import torch

from . import binding as B
from . import layer, mx
from .layer import _on


class Normed(NamedTuple):
    r: torch.Tensor | None            # residual stream after the block (None without y)
    n: torch.Tensor | None            # the next block's input (None without w_pre)
    rstd_post: torch.Tensor | None    # [T] float32, for the backward
    rstd_pre: torch.Tensor | None


def _flags(t, gate, w_post, w_pre):
    """Flags of a norm call; the gate's kind goes by its shape: [d], [T, 1] or [T, d]."""
    T, d = t.shape
    fl = B.dtype_flag(t)
    if w_post is not None:
        fl |= B.MOE_NORM_POST
    if w_pre is not None:
        fl |= B.MOE_NORM_PRE
    if gate is not None:
        kinds = {(T, 1): B.MOE_GATE_TOKEN, (d,): B.MOE_GATE_CHANNEL,
                 (T, d): B.MOE_GATE_TOKEN | B.MOE_GATE_CHANNEL}
        if tuple(gate.shape) not in kinds:
            raise ValueError("gate: %s is none of [d], [T, 1], [T, d] for [%d, %d]" %
                             (tuple(gate.shape), T, d))
        fl |= kinds[tuple(gate.shape)]
    return fl


def _at(t):
    return None if t is None else t.data_ptr()


def norm_forward(res, y=None, gate=None, w_post=None, w_pre=None, res_scale: float = 1.0,
                 eps: float = 1e-6, keep: bool = True, stream=None) -> Normed:
    """r = res_scale * res + gate * post_norm(y), n = pre_norm(r) (moe_norm_fwd). ``res``,
    ``y`` [T, d]; ``gate`` [d], [T, 1], [T, d] or None; ``w_post``, ``w_pre`` [d], None
    where that norm is off. Without ``y``: n = pre_norm(res). ``keep`` False (inference)
    leaves out what only the backward needs."""
    if stream is not None:
        with _on(stream):
            return norm_forward(res, y, gate, w_post, w_pre, res_scale, eps, keep)
    T, d = res.shape
    if y is not None and y.shape != res.shape:
        raise ValueError("y: %s, res is %s" % (tuple(y.shape), tuple(res.shape)))
    fl, el, dev, empty = _flags(res, gate, w_post, w_pre), res.dtype, res.device, torch.empty
    ins = B._args(B._current(), (res, 0, el, "res"), (y, 0, el, "y"), (gate, 0, el, "gate"),
                  (w_post, d, el, "w_post"), (w_pre, d, el, "w_pre"))
    r = n = po = pr = None
    if y is not None:
        r = empty((T, d), dtype=el, device=dev)
    if w_pre is not None:
        n = empty((T, d), dtype=el, device=dev)
    if keep and w_post is not None:
        po = empty(T, dtype=torch.float32, device=dev)
    if keep and w_pre is not None:
        pr = empty(T, dtype=torch.float32, device=dev)
    B._check(B.load_library().moe_norm_fwd(*ins, res_scale, eps, T, d, fl, _at(r), _at(n), _at(po), _at(pr),
                                           B._stream(None)))
    return Normed(r, n, po, pr)


def norm_backward(dr, dn, y, r, rstd_post, rstd_pre, gate=None, w_post=None, w_pre=None,
                  res_scale: float = 1.0, block: bool = True, stream=None):
    """The gradient of norm_forward (moe_norm_bwd): dict(dres, dy, dgate, dw_post, dw_pre),
    None where there is none. ``dr``, ``dn``: gradients of r and n (``dr`` None: only n is
    used further; ``dn`` None without ``w_pre``). ``r``: the forward's, or ``res`` where it
    had no ``y`` (``block`` False). dw_post, dw_pre and a channel's or token's dgate are
    float32, the rest of the inputs' type."""
    if stream is not None:
        with _on(stream):
            return norm_backward(dr, dn, y, r, rstd_post, rstd_pre, gate, w_post, w_pre, res_scale, block)
    t = dr if dr is not None else dn
    if t is None:
        raise ValueError("neither dr nor dn")
    T, d = t.shape
    for v, name in ((dr, "dr"), (dn, "dn"), (y, "y"), (r, "r")):
        if v is not None and v.shape != t.shape:
            raise ValueError("%s: %s, expected %s" % (name, tuple(v.shape), tuple(t.shape)))
    fl, el, dev, f32, empty = _flags(t, gate, w_post, w_pre), t.dtype, t.device, torch.float32, torch.empty
    ins = B._args(B._current(), (dr, 0, el, "dr"), (dn, 0, el, "dn"), (y, 0, el, "y"), (r, 0, el, "r"),
                  (gate, 0, el, "gate"), (w_post, d, el, "w_post"), (w_pre, d, el, "w_pre"),
                  (rstd_post, T, f32, "rstd_post"), (rstd_pre, T, f32, "rstd_pre"))
    dres = empty((T, d), dtype=el, device=dev)
    dy = dgate = dwo = dwr = None
    if block:
        dy = empty((T, d), dtype=el, device=dev)
    if gate is not None:
        dgate = empty(gate.shape, dtype=el if gate.shape == t.shape else f32, device=dev)
    if w_post is not None:
        dwo = empty(d, dtype=f32, device=dev)
    if w_pre is not None:
        dwr = empty(d, dtype=f32, device=dev)
    wsb = B.moe_norm_bwd_workspace_size(T, d, fl)
    ws = empty(max(wsb, 16), dtype=torch.uint8, device=dev)
    B._check(B.load_library().moe_norm_bwd(*ins, res_scale, T, d, fl, dres.data_ptr(), _at(dy), _at(dgate),
                                           _at(dwo), _at(dwr), ws.data_ptr(), wsb, B._stream(None)))
    return dict(dres=dres, dy=dy, dgate=dgate, dw_post=dwo, dw_pre=dwr)


@dataclass
class Block:
    """One block's parameters. ``gate``: [d] or None; ``w_post``: [d] or None. ``experts``:
    the 4-bit experts of ``infer`` (mx.quantize_experts of w1, w3, w2, which ``infer`` does
    not need then)."""
    w_pre: torch.Tensor
    w_gate: torch.Tensor
    w1: torch.Tensor | None = None
    w3: torch.Tensor | None = None
    w2: torch.Tensor | None = None
    k: int = 2
    renorm: bool = False
    bias: torch.Tensor | None = None
    act: str = "swiglu"
    gate: torch.Tensor | None = None
    w_post: torch.Tensor | None = None
    res_scale: float = 1.0
    experts: mx.MXExperts | None = None


@dataclass
class Saved:
    """What forward keeps for backward, block by block."""
    eps: float
    x: torch.Tensor                                # the stream that came in
    n: list = field(default_factory=list)          # each block's normalised input
    rstd: list = field(default_factory=list)       # ... and its reciprocal deviations
    layers: list = field(default_factory=list)     # layer.Saved
    y: list = field(default_factory=list)
    r: list = field(default_factory=list)          # the stream behind each block
    rstd_post: list = field(default_factory=list)


def forward(blocks, x, eps: float = 1e-6, stream=None, **options):
    """x [T, d] through the blocks: (x', saved). ``options`` go to layer.forward (recompute,
    h_on_load, chunk_tokens, atomic_combine)."""
    blocks = list(blocks)
    if not blocks:
        raise ValueError("no blocks")
    with _on(stream):
        s = Saved(eps, x)
        first = norm_forward(x, w_pre=blocks[0].w_pre, eps=eps)
        r, n, rstd = x, first.n, first.rstd_pre
        for i, b in enumerate(blocks):
            y, saved = layer.forward(n, b.w_gate, b.bias, b.w1, b.w3, b.w2, b.k, b.renorm, act=b.act,
                                     **options)
            nxt = blocks[i + 1].w_pre if i + 1 < len(blocks) else None
            o = norm_forward(r, y, b.gate, b.w_post, nxt, b.res_scale, eps)
            s.n.append(n)
            s.rstd.append(rstd)
            s.layers.append(saved)
            s.y.append(y)
            s.r.append(o.r)
            s.rstd_post.append(o.rstd_post)
            r, n, rstd = o.r, o.n, o.rstd_pre
    return r, s


def backward(blocks, saved: Saved, dr, stream=None):
    """Gradients of forward, given that of its result: (dx, [dict for each block]) with
    dw_pre, dw_post, dgate and layer.backward's (dx left out). As layer.backward it
    overwrites the saved A and B."""
    blocks, s = list(blocks), saved
    if len(blocks) != len(s.layers):
        raise ValueError("%d blocks, saved of %d" % (len(blocks), len(s.layers)))
    out = [None] * len(blocks)
    with _on(stream):
        dn = None
        for i in range(len(blocks) - 1, -1, -1):
            b, last = blocks[i], i + 1 == len(blocks)
            o = norm_backward(dr, dn, s.y[i], s.r[i], s.rstd_post[i], None if last else s.rstd[i + 1],
                              b.gate, b.w_post, None if last else blocks[i + 1].w_pre, b.res_scale)
            if not last:
                out[i + 1]["dw_pre"] = o["dw_pre"]
            g = layer.backward(s.layers[i], o["dy"], s.n[i], b.w_gate, b.w1, b.w3, b.w2)
            dn, dr = g.pop("dx"), o["dres"]
            out[i] = dict(g, dgate=o["dgate"], dw_post=o["dw_post"])
        o = norm_backward(dr, dn, None, s.x, None, s.rstd[0], w_pre=blocks[0].w_pre, block=False)
        out[0]["dw_pre"] = o["dw_pre"]
    return o["dres"], out


def infer(blocks, x, eps: float = 1e-6, rows: str = "bf16", stream=None):
    """x (bfloat16) through the blocks with their 4-bit ``experts`` (mx.forward); nothing is
    kept."""
    blocks = list(blocks)
    if not blocks:
        raise ValueError("no blocks")
    if any(b.experts is None for b in blocks):
        raise ValueError("a block has no 4-bit experts (mx.quantize_experts)")
    with _on(stream):
        r, n = x, norm_forward(x, w_pre=blocks[0].w_pre, eps=eps, keep=False).n
        for i, b in enumerate(blocks):
            y = mx.forward(n, b.w_gate, b.bias, b.experts, b.k, b.renorm, b.act, rows)
            nxt = blocks[i + 1].w_pre if i + 1 < len(blocks) else None
            o = norm_forward(r, y, b.gate, b.w_post, nxt, b.res_scale, eps, keep=False)
            r, n = o.r, o.n
    return r
