"""The global norm of gradients, and clipping by it, over any list of contiguous tensors,
which may start anywhere: the layer's own gradients are float32, a model's others may be
bfloat16."""
from __future__ import annotations

import torch

from . import binding as B
from .layer import _on

# what layer.backward gives beside the gradients of parameters
NOT_PARAMETERS = ("dx", "dX_slot", "dx_ffn", "d_gates")


def _list(grads):
    """The tensors of a list or tuple, without None; of a dict, as layer.backward returns, or of
    dicts in the list, as block.backward's, the gradients of parameters."""
    if isinstance(grads, dict):
        return [g for n, g in grads.items() if g is not None and n not in NOT_PARAMETERS]
    grads = [g for g in grads if g is not None]
    if dict in map(type, grads):
        return [t for g in grads for t in (_list(g) if isinstance(g, dict) else (g,))]
    return grads


def _norm(tl):
    dev = _device(tl)
    norm = torch.empty((), dtype=torch.float32, device=dev)
    sumsq = torch.empty((), dtype=torch.float64, device=dev)
    wsb = B.moe_grad_norm_workspace_size(tl.n)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device=dev)
    B._check(B.load_library().moe_grad_norm(*tl.addresses(), tl.n, sumsq.data_ptr(), norm.data_ptr(),
                                            ws.data_ptr(), wsb, B._stream(None)))
    return norm, sumsq


def _device(tl):
    return tl.tensors[0].device if tl.n else torch.device("cuda", torch.cuda.current_device())


def norm(grads, stream=None):
    """(norm, sumsq): the 2-norm over all elements of all tensors, float32, and its square,
    float64, both on the GPU. ``grads``: tensors, or the dict (dicts) of layer.backward
    (block.backward), whose NOT_PARAMETERS stay out. Where a model's gradients are spread over
    several devices the devices' sumsq add up."""
    with _on(stream):
        return _norm(B.TensorList(_list(grads)))


def clip(grads, max_norm: float, out=None, sumsq=None, stream=None):
    """Scale the gradients (as in ``norm``) by min(1, max_norm / (norm + 1e-6)), in place or
    into ``out`` (tensors of the same sizes and types, in the same order). ``sumsq``: the
    square of the norm to go by (a float64 GPU tensor: the sum over several devices'),
    None: these tensors' own. ``max_norm`` infinite: the norm alone is of use, nothing is
    scaled. Returns the norm, on the GPU; nothing waits for the host."""
    with _on(stream):
        tl = B.TensorList(_list(grads))
        outs = None if out is None else B.TensorList(_list(out))
        if outs is not None and outs.n != tl.n:
            raise ValueError("out: %d tensors for %d gradients" % (outs.n, tl.n))
        if sumsq is None:
            total, sumsq = _norm(tl)
        else:
            total = sumsq.sqrt().float()
        B.moe_grad_clip(tl, outs, sumsq, max_norm, None)
    return total
