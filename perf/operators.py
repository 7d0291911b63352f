"""The measured work of the operators around the MoE layer: the norms of a residual
block, the gradient norm with clipping, microscaled 4-bit (MXFP4) quantisation, and
the grouped products over experts held in it.

Sizes are those of ``synth.CONFIGS`` and the paper's Table 1 shapes; row counts run
from one decoded token to a full training batch. ``run`` computes the plain form in
torch, or, with ``own``, makes the framework's calls on the same tensors.
"""
import math

import numpy as np
import torch

own = False

# (d, f, E, k): layer shapes of the repository's workloads and sweeps
MID = (2048, 1408, 64, 6)
FEW_LARGE = (4096, 14336, 8, 2)
MANY_SMALL = (2048, 768, 128, 8)
WIDE = (4096, 2048, 64, 8)
ODD = (2880, 2880, 128, 4)
CONF1 = (512, 2048, 4, 1)
CONF6 = (1024, 4096, 16, 4)
CONF7 = (2048, 8192, 8, 4)
TINY = (256, 512, 8, 2)
SHAPES = (MID, FEW_LARGE, MANY_SMALL, WIDE, ODD, CONF1, CONF6, CONF7, TINY)

EPS = 1e-6
MOST_FLOPS = 1.0e12     # of a drawn product
MOST_ELEMENTS = 1.2e8   # of a drawn norm
MOST_GRADS = 5.6e8      # elements of a drawn gradient list


def _quant(name, rows, K, batch=1, transpose=False, dtype="bf16"):
    return _named(name, dict(op="quantize", batch=batch, rows=rows, K=K, transpose=transpose, dtype=dtype))


def _prod(name, T, shape, first, act, x4, zipf=0.0):
    """first: the gathered d -> f product; else f -> d over the slots' own rows.
    x4: the rows are microscaled 4-bit too, else bfloat16."""
    d, f, E, k = shape
    return _named(name, dict(op="product", T=T, K=d if first else f, N=f if first else d, E=E, k=k,
                             gather=first, act=act, x4=x4, zipf=zipf))


def _norm(name, op, T, d, dtype="bf16", post=True, pre=True, gate="channel", scale=1.0):
    return _named(name, dict(op=op, T=T, d=d, dtype=dtype, post=post, pre=pre, gate=gate, scale=scale))


def _clip(name, shape, layers, dtype="f32", max_norm=1.0, big=True):
    """Gradients of ``layers`` layers: the experts' (big) and the router's, two norms'
    and a gate's, or only the small ones."""
    d, f, E, _ = shape
    return _named(name, dict(op="clip", d=d, f=f, E=E, layers=layers, dtype=dtype, max_norm=max_norm, big=big))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # the rows of a decode batch between two 4-bit products
        _quant("quantize_rows_48", 48, 2048),
        # a layer's expert weights when a trained model is made ready for serving: [E, d, f]
        # quantised along d, the axis that the product sums over
        _quant("quantize_weights_mid", 1408, 2048, batch=64, transpose=True),
        # generating one sequence: one token's two experts, the gated first product
        _prod("product_decode_1", 1, FEW_LARGE, True, "swiglu", False),
        # a busy server's decode batch, the down product over ragged slots, odd widths
        _prod("product_decode_odd_300", 300, ODD, False, "none", False),
        # prompts of a server with rows in 4 bits too: few large experts
        _prod("product_prefill_1777", 1777, FEW_LARGE, True, "swiglu", True),
        # a long batch of prompts (scoring, distillation) over many experts, bfloat16 rows
        _prod("product_batch_16384", 16384, MID, True, "swiglu", False),
        # decode: the tail of one block and the head of the next, one launch
        _norm("norm_decode_48", "norm_fwd", 48, 2048),
        # training at the headline width: forward over a full batch
        _norm("norm_fwd_32768", "norm_fwd", 32768, 4096),
        # its backward, with an odd token count and a token-wise gate
        _norm("norm_bwd_16383", "norm_bwd", 16383, 4096, gate="token", scale=0.7),
        # float32 numerics debugging of a small block, backward
        _norm("norm_bwd_f32_1021", "norm_bwd", 1021, 2880, dtype="f32", gate="channel"),
        # the small parameters of a dozen layers: many tensors, little data
        _clip("clip_small_12", MID, 12, big=False),
        # one layer's gradients after its backward: three of the experts' matrices and the rest
        _clip("clip_mid", MID, 1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: rows from 1 to a full batch, widths of the repository's shapes or
    any multiple of what an operator takes."""
    op = rng.choice(["quantize", "product", "product", "product", "norm_fwd", "norm_bwd", "clip"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d, f, E, k = shape = rng.choice(SHAPES)
    if op == "quantize":
        if rng.random() < 0.5:
            return _quant(None, _log_int(rng, 1, 32768), 32 * _log_int(rng, 1, 160), dtype=dtype)
        K, R = rng.choice([(d, f), (f, d)])
        return _quant(None, R, K, batch=rng.randint(1, max(1, min(E, int(1.8e8 / (K * R))))),
                      transpose=True, dtype=dtype)
    if op == "product":
        first = rng.random() < 0.6
        act = rng.choice(["swiglu", "swiglu", "silu", "relu", "none"]) if first else "none"
        per = 2.0 * k * d * f * (2 if act == "swiglu" else 1)
        T = _log_int(rng, 1, max(2, min(32768, MOST_FLOPS / per)))
        return _prod(None, T, shape, first, act, rng.random() < 0.5, rng.choice([0.0, 0.0, 1.2]))
    if op == "clip":
        big = rng.random() < 0.5
        most = int(MOST_GRADS / (3.0 * E * d * f)) if big else 12
        if most < 1:
            d, f, E, k = shape = TINY
            most = 12
        return _clip(None, shape, rng.randint(1, min(most, 7 if big else 12)), dtype,
                     rng.choice([0.5, 1.0, 1e6]), big)
    d = rng.choice([d, 8 * _log_int(rng, 8, 1024)])
    post, pre = rng.choice([(True, True), (True, True), (True, False), (False, True)])
    return _norm(None, op, _log_int(rng, 1, min(65536, MOST_ELEMENTS / d)), d, dtype, post, pre,
                 rng.choice(["none", "channel", "channel", "token", "full"]),
                 rng.choice([1.0, 1.0, 0.7]))


# ---- inputs -------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _normal(gen, shape, std, dt):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dt)


def _codes(gen, shape, std):
    """Random weights or rows as a program holds them in microscaled 4 bits: codes
    [..., K/2] and scale bytes [..., K/32], from normal values of that deviation."""
    x = torch.randn((*shape[:-1], shape[-1] // 32, 32), generator=gen, device="cuda").mul_(std)
    e = torch.frexp(x.abs().amax(-1, keepdim=True))[1] - 3
    idx = torch.bucketize(torch.ldexp(x.abs(), -e), _mids(x.device)).clamp_(max=7).to(torch.uint8)
    idx += (x < 0).to(torch.uint8) * 8
    idx = idx.reshape(*shape[:-1], shape[-1] // 2, 2)
    return (idx[..., 0] + idx[..., 1] * 16).contiguous(), (e[..., 0] + 127).to(torch.uint8)


def _mids(device):
    return torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=device)


def _prepare_product(c, seed):
    """x ~ N(0, 1) (the slots' own rows: of the size of a gated hidden row, 0.4), weights
    N(0, 1/sqrt(K)); routing: the top k of random scores, with a Zipf bias or none, and the
    maps that moe_build_index gives: slots by expert, tokens ascending in each."""
    gen = _generator(seed)
    T, E, k, K, N = c["T"], c["E"], c["k"], c["K"], c["N"]
    score = torch.rand((T, E), generator=gen, device="cuda").log_().neg_().log_().neg_()
    if c["zipf"]:
        rank = torch.from_numpy(np.random.Generator(np.random.PCG64(seed)).permutation(E) + 1.0)
        score -= (c["zipf"] * rank.log()).to(score)
    ids = score.topk(k, 1).indices.reshape(-1)
    slot = torch.sort(ids, stable=True).indices
    counts = torch.bincount(ids, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    rows = (slot // k).to(torch.int32)
    n = T if c["gather"] else T * k
    std = 1.0 if c["gather"] else 0.4
    x = _codes(gen, (n, K), std) if c["x4"] else _normal(gen, (n, K), std, torch.bfloat16)
    w = [torch.cat(p) for p in zip(*(_codes(gen, (1, N, K), K ** -0.5) for _ in range(E)))]
    w3 = None
    if c["act"] == "swiglu":
        w3 = [torch.cat(p) for p in zip(*(_codes(gen, (1, N, K), K ** -0.5) for _ in range(E)))]
    return dict(x=x, w=w, w3=w3, offsets=offsets, rows=rows if c["gather"] else None,
                bounds=offsets.tolist())


def _prepare_norm(c, seed):
    """Residual rows of growing size, block outputs ~ N(0, 1), norm weights near one; for
    the backward the forward's r and reciprocal deviations, and N(0, 1) gradients."""
    gen, dt, T, d = _generator(seed), _type(c), c["T"], c["d"]
    s = dict(res=_normal(gen, (T, d), 3.0, dt), y=_normal(gen, (T, d), 1.0, dt), gate=None,
             w_post=None, w_pre=None, scale=c["scale"])
    shape = dict(none=None, channel=(d,), token=(T, 1), full=(T, d))[c["gate"]]
    if shape is not None:
        s["gate"] = (torch.rand(shape, generator=gen, device="cuda") * 0.9 + 0.1).to(dt)
    if c["post"]:
        s["w_post"] = (1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    if c["pre"]:
        s["w_pre"] = (1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    if c["op"] == "norm_bwd":
        r, _, rstd_post, rstd_pre = _plain_norm_fwd(s)
        s.update(r=r, rstd_post=rstd_post, rstd_pre=rstd_pre, dr=_normal(gen, (T, d), 1.0, dt),
                 dn=_normal(gen, (T, d), 1.0, dt) if c["pre"] else None)
    return s


def _prepare_clip(c, seed):
    gen, dt = _generator(seed), _type(c)
    d, f, E = c["d"], c["f"], c["E"]
    shapes = [(E, d), (d,), (d,), (d,)]
    if c["big"]:
        shapes = [(E, d, f), (E, d, f), (E, f, d)] + shapes
    grads = [_normal(gen, s, 0.01, dt) for _ in range(c["layers"]) for s in shapes]
    return dict(grads=grads, outs=[torch.empty_like(g) for g in grads], max_norm=c["max_norm"])


def prepare(case, seed):
    c = case
    if c["op"] == "quantize":
        # a few channels ten times the others, as activations and weights have them
        shape = (c["batch"], c["K"], c["rows"]) if c["transpose"] else (c["batch"], c["rows"], c["K"])
        gen = _generator(seed)
        x = torch.randn(shape, generator=gen, device="cuda")
        x *= 1.0 + 9.0 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.01)
        s = dict(x=x.to(_type(c)))
    elif c["op"] == "product":
        s = _prepare_product(c, seed)
    elif c["op"] == "clip":
        s = _prepare_clip(c, seed)
    else:
        s = _prepare_norm(c, seed)
    s["case"] = c
    return s


# ---- the plain forms ------------------------------------------------------------------------

def _plain_quantize(x, transpose):
    """Scale 2^(floor(log2(largest)) - 2) for each 32 values along K, each value to the
    nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code); the values they stand for."""
    v = x.transpose(-1, -2) if transpose else x
    v = v.float().unflatten(-1, (-1, 32))
    e = torch.frexp(v.abs().amax(-1, keepdim=True))[1] - 3
    a = torch.ldexp(v.abs(), -e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp_(max=6.0)
    return torch.ldexp(a * v.sign(), e).flatten(-2).to(x.dtype)


def _plain_values(codes, scales):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
    s = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    return (v.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _plain_product(s):
    c, o = s["case"], s["bounds"]
    x = _plain_values(*s["x"]) if c["x4"] else s["x"].float()
    if c["gather"]:
        x = x[s["rows"].long()]

    def grouped(w):
        return torch.cat([x[o[e]:o[e + 1]] @ _plain_values(w[0][e], w[1][e]).t()
                          for e in range(c["E"]) if o[e + 1] > o[e]])

    a = grouped(s["w"])
    if c["act"] == "relu":
        a = a.clamp_min(0.0)
    elif c["act"] != "none":
        a = a / (1.0 + torch.exp(-a))
    if c["act"] == "swiglu":
        a = a * grouped(s["w3"])
    return a.to(torch.bfloat16)


def _plain_norm_fwd(s):
    dt = s["y"].dtype
    p, rstd_post, n, rstd_pre = s["y"].float(), None, None, None
    if s["w_post"] is not None:
        rstd_post = torch.rsqrt(p.square().mean(1) + EPS)
        p = p * rstd_post[:, None] * s["w_post"].float()
    if s["gate"] is not None:
        p = p * s["gate"].float()
    r = s["scale"] * s["res"].float() + p
    if s["w_pre"] is not None:
        rstd_pre = torch.rsqrt(r.square().mean(1) + EPS)
        n = (r * rstd_pre[:, None] * s["w_pre"].float()).to(dt)
    return r.to(dt), n, rstd_post, rstd_pre


def _plain_norm_bwd(s):
    dt, y = s["y"].dtype, s["y"].float()
    out = {}
    G = s["dr"].float()
    if s["w_pre"] is not None:
        hat, dn = s["r"].float() * s["rstd_pre"][:, None], s["dn"].float()
        out["dw_pre"] = (dn * hat).sum(0)
        dn = dn * s["w_pre"].float()
        G = G + s["rstd_pre"][:, None] * (dn - hat * (dn * hat).mean(1, keepdim=True))
    out["dres"] = (s["scale"] * G).to(dt)
    p = hat = y
    if s["w_post"] is not None:
        hat = y * s["rstd_post"][:, None]
        p = hat * s["w_post"].float()
    dp = G
    if s["gate"] is not None:
        kind = s["case"]["gate"]
        dg = G * p
        out["dgate"] = dg.sum(0) if kind == "channel" else dg.sum(1, keepdim=True) if kind == "token" else dg.to(dt)
        dp = G * s["gate"].float()
    if s["w_post"] is not None:
        out["dw_post"] = (dp * hat).sum(0)
        dp = dp * s["w_post"].float()
        dp = s["rstd_post"][:, None] * (dp - hat * (dp * hat).mean(1, keepdim=True))
    out["dy"] = dp.to(dt)
    return out


def _plain_clip(s):
    total = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    scale = (s["max_norm"] / (total + 1e-6)).clamp(max=1.0).float()
    return [total.float()] + [(g.float() * scale).to(g.dtype) for g in s["grads"]]


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    if c["op"] == "quantize":
        return _plain_quantize(s["x"], c["transpose"])
    if c["op"] == "product":
        return _plain_product(s)
    if c["op"] == "clip":
        return _plain_clip(s)
    if c["op"] == "norm_bwd":
        return _plain_norm_bwd(s)
    return [t for t in _plain_norm_fwd(s) if t is not None]


def _own(s, c):
    from paper_2601_05296_amd import block, grads, mx
    if c["op"] == "quantize":
        return mx.dequantize(mx.quantize(s["x"], transpose=c["transpose"]), s["x"].dtype)
    if c["op"] == "product":
        x = mx.MX(*s["x"]) if c["x4"] else s["x"]
        w3 = None if s["w3"] is None else mx.MX(*s["w3"])
        return mx.product(x, mx.MX(*s["w"]), s["offsets"], rows=s["rows"], w3=w3, act=c["act"])
    if c["op"] == "clip":
        return [grads.clip(s["grads"], s["max_norm"], out=s["outs"])] + s["outs"]
    if c["op"] == "norm_bwd":
        g = block.norm_backward(s["dr"], s["dn"], s["y"], s["r"], s["rstd_post"], s["rstd_pre"],
                                gate=s["gate"], w_post=s["w_post"], w_pre=s["w_pre"],
                                res_scale=s["scale"])
        return {n: t for n, t in g.items() if t is not None}
    got = block.norm_forward(s["res"], s["y"], gate=s["gate"], w_post=s["w_post"], w_pre=s["w_pre"],
                             res_scale=s["scale"], eps=EPS)
    return [t for t in got if t is not None]


# ---- what a pass needs -------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "quantize":
        n, el = c["batch"] * c["rows"] * c["K"], 4 if c["dtype"] == "f32" else 2
        # the values in, the codes and scales out and in again, the values they stand for out
        return dict(bytes=int(n * (2 * el + 2 * 17 / 32)), flops=6 * n)
    if c["op"] == "product":
        T, K, N, E, k = c["T"], c["K"], c["N"], c["E"], c["k"]
        mats = 2 if c["act"] == "swiglu" else 1
        active = E * (1.0 - (1.0 - k / E) ** T)
        n = T if c["gather"] else T * k
        byts = mats * active * N * K * 17 / 32 + n * K * (17 / 32 if c["x4"] else 2) + T * k * (N * 2 + 4)
        return dict(bytes=int(byts), flops=int(2 * mats * T * k * N * K))
    if c["op"] == "clip":
        d, f, E = c["d"], c["f"], c["E"]
        n = c["layers"] * (E * d + 3 * d + (3 * E * d * f if c["big"] else 0))
        return dict(bytes=2 * n * (4 if c["dtype"] == "f32" else 2), flops=3 * n)
    n, el = c["T"] * c["d"], 4 if c["dtype"] == "f32" else 2
    fwd = c["op"] == "norm_fwd"
    tensors = 3 + c["pre"] if fwd else 3 + 2 * c["pre"] + (c["post"] or c["gate"] != "none")
    if c["gate"] == "full":
        tensors += 1 if fwd else 2
    return dict(bytes=int(n * el * tensors), flops=(10 if fwd else 25) * n)


# ---- 64 bits -----------------------------------------------------------------------------------

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_quantize(c, s):
    """By the borders between neighbouring values."""
    x = s["x"].double()
    x = (x.transpose(1, 2) if c["transpose"] else x).reshape(-1, 32)
    top = x.abs().max(1, keepdim=True).values
    # floor(log2(top)) from the bits of the (normal) 64-bit value; a block of zeros has scale 1
    e = ((top.view(torch.int64) >> 52) - 1023 - 2) * (top > 0)
    unit = ((e + 1023) << 52).view(torch.float64)
    q = x.abs() / unit
    # value lo + 1 from its lower border on; the border itself goes to the even one of its two codes
    v = sum((_E2M1[lo + 1] - _E2M1[lo]) * (q >= b if lo % 2 else q > b).double()
            for lo, b in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    v = (v * unit).copysign(x)
    return v.reshape(c["batch"], c["rows"], c["K"])


def _exact_values(codes, scales):
    """Each value from its code's sign, exponent and mantissa bits."""
    code = torch.stack((codes.to(torch.int64) % 16, codes.to(torch.int64) // 16), -1).flatten(-2)
    sign, ex, man = 1.0 - 2.0 * (code // 8), code // 2 % 4, code % 2
    v = torch.where(ex == 0, 0.5 * man, (1.0 + 0.5 * man) * 2.0 ** (ex - 1).double())
    return sign * v * 2.0 ** (scales.double() - 127.0).repeat_interleave(32, -1)


def _exact_product(c, s):
    x = _exact_values(*s["x"]) if c["x4"] else s["x"].double()
    if c["gather"]:
        x = x.index_select(0, s["rows"])

    def expert(e):
        rows = x[s["bounds"][e]:s["bounds"][e + 1]]
        a = rows @ _exact_values(s["w"][0][e], s["w"][1][e]).t()
        if c["act"] == "relu":
            return torch.where(a > 0, a, 0.0)
        if c["act"] == "none":
            return a
        h = a * torch.sigmoid(a)
        if c["act"] == "swiglu":
            h = h * (rows @ _exact_values(s["w3"][0][e], s["w3"][1][e]).t())
        return h

    return torch.cat([expert(e) for e in range(c["E"]) if s["bounds"][e + 1] > s["bounds"][e]])


def _exact_norm_fwd(c, s):
    y, res = s["y"].double(), s["res"].double()
    got, p = [], y
    if c["post"]:
        sd = (y.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt()
        p = y / sd * s["w_post"].double()
        got.append(1.0 / sd[:, 0])
    if c["gate"] != "none":
        p = s["gate"].double() * p
    r = c["scale"] * res + p
    if not c["pre"]:
        return [r] + got
    sd = (r.pow(2).sum(1, keepdim=True) / c["d"] + EPS).sqrt()
    return [r, r / sd * s["w_pre"].double()] + got + [1.0 / sd[:, 0]]


def _exact_norm_bwd(c, s):
    """By the chain rule on row vectors: for v = w u / sd(u), du = (w dv - u <w dv, u> / (d sd^2)) / sd,
    with the reciprocal deviations as they are given."""
    d, y, r = c["d"], s["y"].double(), s["r"].double()
    G, out = s["dr"].double(), {}

    def through(dv, u, w, rstd):
        i = rstd.double()[:, None]
        wd = w.double() * dv
        return i * wd - u * (i ** 3 / d) * (wd * u).sum(1, keepdim=True)

    if c["pre"]:
        dn = s["dn"].double()
        out["dw_pre"] = torch.einsum("td,td,t->d", dn, r, s["rstd_pre"].double())
        G = G + through(dn, r, s["w_pre"], s["rstd_pre"])
    out["dres"] = c["scale"] * G
    i = s["rstd_post"].double()[:, None] if c["post"] else 1.0
    w = s["w_post"].double() if c["post"] else 1.0
    dp = G
    if c["gate"] != "none":
        full = G * y * i * w
        out["dgate"] = dict(channel=lambda: full.sum(0), token=lambda: full.sum(1)[:, None],
                            full=lambda: full)[c["gate"]]()
        dp = G * s["gate"].double()
    if c["post"]:
        out["dw_post"] = (dp * y * i).sum(0)
        dp = through(dp, y, s["w_post"], s["rstd_post"])
    out["dy"] = dp
    return out


def _exact_clip(c, s):
    norm = math.sqrt(sum(float(torch.linalg.vecdot(p.double(), p.double()))
                         for g in s["grads"] for p in g.reshape(-1).split(1 << 26)))
    k = min(1.0, c["max_norm"] / (norm + 1e-6))
    return [torch.tensor(norm, dtype=torch.float64)] + [g.double() * k for g in s["grads"]]


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    c, s = case, prepare(case, seed)
    return dict(quantize=_exact_quantize, product=_exact_product, clip=_exact_clip,
                norm_fwd=_exact_norm_fwd, norm_bwd=_exact_norm_bwd)[c["op"]](c, s)
