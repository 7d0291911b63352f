"""CPU checks of the operators around the layer: their refusals, before anything reaches
the GPU, and the 64-bit forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import block, grads, mx
from tests import block_ref as R

FAKE = 1 << 20   # aligned, never dereferenced
INV, UNS, WSP = B.MOE_ERR_INVALID_ARG, B.MOE_ERR_UNSUPPORTED, B.MOE_ERR_WORKSPACE


def _fwd(res=FAKE, y=FAKE, gate=None, w_post=None, w_pre=None, scale=1.0, eps=1e-6, T=4, d=64,
         flags=0, r=2 * FAKE, n=None):
    return B.load_library().moe_norm_fwd(res, y, gate, w_post, w_pre, scale, eps, T, d, flags, r, n,
                                         None, None, None)


@pytest.mark.parametrize("kw,status,what", [
    (dict(d=0), INV, b"d = 0"), (dict(d=12), UNS, b"multiple of 8"), (dict(d=8200), UNS, b"8192"),
    (dict(T=-1), INV, b"T = -1"), (dict(flags=B.MOE_RENORM), INV, b"unknown flag"),
    (dict(eps=0.0), INV, b"eps"), (dict(eps=float("nan")), INV, b"eps"),
    (dict(scale=float("inf")), INV, b"res_scale"),
    (dict(res=None), INV, b"res is NULL"), (dict(res=FAKE + 8), INV, b"aligned"),
    (dict(r=None), INV, b"r is NULL"), (dict(gate=FAKE), INV, b"gate without"),
    (dict(w_pre=FAKE), INV, b"w_pre without"), (dict(flags=B.MOE_NORM_POST), INV, b"w_post is NULL"),
    (dict(flags=B.MOE_NORM_PRE, w_pre=FAKE), INV, b"n is NULL"),
    (dict(flags=B.MOE_NORM_PRE, w_pre=FAKE, n=2 * FAKE), INV, b"the same"),
    (dict(y=None, r=None), INV, b"nothing to do"),
    (dict(y=None, r=None, flags=B.MOE_NORM_PRE | B.MOE_GATE_TOKEN, gate=FAKE, w_pre=FAKE, n=FAKE), INV,
     b"without a block output"),
    (dict(y=None, r=None, scale=0.5, flags=B.MOE_NORM_PRE, w_pre=FAKE, n=FAKE), INV, b"res_scale"),
    (dict(y=None, flags=B.MOE_NORM_PRE, w_pre=FAKE, n=3 * FAKE), INV, b"r without"),
])
def test_norm_fwd_refusals(kw, status, what):
    assert _fwd(**kw) == status and what in B.load_library().moe_last_error()


def test_norm_fwd_no_rows():
    assert _fwd(T=0, res=None, y=None, r=None) == B.MOE_OK


def _bwd(dr=FAKE, dn=None, y=None, r=None, gate=None, w_post=None, w_pre=None, po=None, pr=None,
         scale=1.0, T=4, d=64, flags=0, dres=FAKE, dy=2 * FAKE, dgate=None, dwo=None, dwr=None,
         ws=FAKE, wsb=1 << 40):
    return B.load_library().moe_norm_bwd(dr, dn, y, r, gate, w_post, w_pre, po, pr, scale, T, d, flags,
                                         dres, dy, dgate, dwo, dwr, ws, wsb, None)


POST = dict(flags=B.MOE_NORM_POST, w_post=FAKE, dwo=FAKE, po=FAKE, y=FAKE)
PRE = dict(flags=B.MOE_NORM_PRE, w_pre=FAKE, dwr=FAKE, pr=FAKE, r=FAKE, dn=FAKE)


@pytest.mark.parametrize("kw,status,what", [
    (dict(d=20), UNS, b"multiple of 8"), (dict(flags=B.MOE_ACCUMULATE), INV, b"unknown flag"),
    (dict(dr=None), INV, b"no gradient comes in"), (dict(dres=None), INV, b"dres is NULL"),
    (dict(dy=FAKE), INV, b"the same"), (dict(dgate=FAKE), INV, b"dgate without"),
    (dict(flags=B.MOE_GATE_CHANNEL, gate=FAKE, dgate=FAKE), INV, b"y is NULL"),
    ({**POST, "y": None}, INV, b"y is NULL"), ({**POST, "po": None}, INV, b"rstd_post is NULL"),
    ({**POST, "dwo": None}, INV, b"dw_post is NULL"), ({**PRE, "dn": None}, INV, b"dn is NULL"),
    ({**PRE, "r": None}, INV, b"r is NULL"), ({**PRE, "pr": None}, INV, b"rstd_pre is NULL"),
    ({**PRE, "dy": None, "scale": 2.0}, INV, b"res_scale"), ({**POST, "dy": None}, INV, b"without a block"),
    ({**PRE, "wsb": 16}, WSP, b"workspace"), ({**PRE, "ws": None}, WSP, b"workspace"),
])
def test_norm_bwd_refusals(kw, status, what):
    assert _bwd(**kw) == status and what in B.load_library().moe_last_error()


def test_norm_workspace_is_bounded():
    """The partial sums do not grow with the rows: at most 512 of 3 d floats, or 2048 rows
    of a narrow one."""
    lib = B.load_library()
    for d in (8, 512, 1024, 4096, 8192):
        for fl in (0, B.MOE_F32):
            n = lib.moe_norm_bwd_workspace_size(1 << 30, d, fl)
            assert 0 < n <= 2048 * 3 * d * 4
            assert lib.moe_norm_bwd_workspace_size(1, d, fl) <= 4 * 3 * d * 4
    assert lib.moe_norm_bwd_workspace_size(0, 64, 0) == 0


def _lists(ptrs, sizes, types):
    n = len(ptrs)
    return ((ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*sizes), (ctypes.c_uint * n)(*types))


def test_grad_refusals():
    lib = B.load_library()

    def norm(ptrs, sizes, types, n=None, sumsq=FAKE, out=FAKE, ws=FAKE, wsb=1 << 30):
        p, s, t = _lists(ptrs, sizes, types)
        return lib.moe_grad_norm(p, s, t, len(ptrs) if n is None else n, sumsq, out, ws, wsb, None)

    def clip(ptrs, outs, sizes, types, max_norm=1.0, sumsq=FAKE):
        p, s, t = _lists(ptrs, sizes, types)
        o = None if outs is None else (ctypes.c_void_p * len(outs))(*outs)
        return lib.moe_grad_clip(p, o, s, t, len(ptrs), sumsq, max_norm, None)

    bf, f32 = B.MOE_BF16, B.MOE_F32
    assert norm([FAKE], [4], [f32], n=-1) == INV
    assert norm([FAKE], [-4], [f32]) == INV and b"sizes[0]" in lib.moe_last_error()
    assert norm([FAKE], [4], [2]) == INV and b"types[0]" in lib.moe_last_error()
    assert norm([None], [4], [f32]) == INV and b"NULL" in lib.moe_last_error()
    assert norm([FAKE + 2], [4], [f32]) == INV and b"aligned" in lib.moe_last_error()
    assert norm([FAKE + 1], [4], [bf]) == INV
    assert norm([FAKE], [4], [f32], sumsq=None) == INV
    assert norm([FAKE], [4], [f32], out=FAKE + 2) == INV
    assert norm([FAKE], [4], [f32], wsb=8) == WSP
    assert norm([FAKE], [4], [f32], ws=None) == WSP
    assert lib.moe_grad_norm(None, None, None, 1, FAKE, FAKE, FAKE, 1 << 30, None) == INV
    assert clip([FAKE], None, [4], [f32], max_norm=-1.0) == INV
    assert clip([FAKE], None, [4], [f32], max_norm=float("nan")) == INV
    assert clip([FAKE], None, [4], [f32], sumsq=None) == INV
    assert clip([FAKE], [None], [4], [f32]) == INV and b"outs[0]" in lib.moe_last_error()
    # written tensors may not share memory with any other of the call
    assert clip([FAKE, FAKE], None, [4, 4], [f32, f32]) == INV and b"overlap" in lib.moe_last_error()
    assert clip([FAKE, FAKE + 8], None, [4, 4], [f32, f32]) == INV
    assert clip([FAKE, FAKE + 64], [2 * FAKE, FAKE + 8], [4, 4], [f32, f32]) == INV
    assert clip([FAKE, FAKE + 64], [2 * FAKE, 2 * FAKE], [4, 4], [f32, f32]) == INV
    assert clip([FAKE, FAKE, 3 * FAKE], [2 * FAKE, 4 * FAKE, 2 * FAKE + 12], [4, 4, 4], [f32] * 3) == INV
    # a large span that reaches behind a small one in between
    assert clip([FAKE, FAKE + 16, FAKE + 64], [FAKE, 2 * FAKE, 3 * FAKE], [64, 0, 4], [f32] * 3) == INV
    # nothing to do: no tensors, or only empty ones
    assert clip([None, None], None, [0, 0], [f32, bf]) == B.MOE_OK
    assert lib.moe_grad_norm_workspace_size(0) == 0 < lib.moe_grad_norm_workspace_size(1)


def test_mx_refusals():
    lib = B.load_library()

    def quant(src=FAKE, batch=1, rows=4, K=64, flags=0, codes=FAKE, scales=FAKE):
        return lib.moe_mx_quantize(src, batch, rows, K, flags, codes, scales, None)

    assert quant(K=48) == UNS and quant(K=0) == INV and quant(rows=-1) == INV and quant(batch=-1) == INV
    assert quant(flags=B.MOE_RENORM) == INV and quant(src=None) == INV and quant(codes=FAKE + 4) == INV
    assert quant(rows=3, flags=B.MOE_TRANSPOSED) == UNS
    assert quant(batch=65536, rows=2, flags=B.MOE_TRANSPOSED) == UNS
    assert quant(rows=1 << 29, K=32, flags=B.MOE_TRANSPOSED) == UNS
    assert quant(rows=2, K=(1 << 24) + 32, flags=B.MOE_TRANSPOSED) == UNS
    assert quant(batch=1 << 20, rows=1 << 20) == UNS
    assert quant(rows=0, src=None) == B.MOE_OK and quant(batch=0, src=None) == B.MOE_OK
    deq = lib.moe_mx_dequantize
    assert deq(FAKE, FAKE, 4, 48, 0, FAKE, None) == UNS and deq(FAKE, FAKE, -1, 64, 0, FAKE, None) == INV
    assert deq(FAKE, FAKE, 4, 64, B.MOE_TRANSPOSED, FAKE, None) == INV
    assert deq(FAKE, None, 4, 64, 0, FAKE, None) == INV and deq(None, None, 0, 64, 0, None, None) == B.MOE_OK


def test_mx_gemm_refusals():
    lib = B.load_library()

    def gemm(x=FAKE, xs=None, w=FAKE, ws=FAKE, w3=None, ws3=None, off=FAKE, rows=FAKE, T=4, S=8, K=64,
             N=64, E=2, flags=0, out=FAKE):
        return lib.moe_mx_gemm(x, xs, w, ws, w3, ws3, off, rows, T, S, K, N, E, flags, out, None)

    assert gemm(K=32) == UNS and gemm(N=96) == UNS and gemm(K=0) == INV
    assert gemm(E=0) == INV and gemm(E=257) == UNS
    assert gemm(flags=B.MOE_F32) == UNS and gemm(flags=B.MOE_RENORM) == INV
    assert gemm(flags=B.MOE_ACT_SILU | B.MOE_ACT_RELU) == INV
    assert gemm(flags=B.MOE_GATED | B.MOE_ACT_RELU, w3=FAKE, ws3=FAKE) == INV
    assert gemm(flags=B.MOE_GATED) == INV and b"w3 is NULL" in lib.moe_last_error()
    assert gemm(flags=B.MOE_GATED, w3=FAKE) == INV and b"w3_scales is NULL" in lib.moe_last_error()
    assert gemm(w3=FAKE) == INV and b"without MOE_GATED" in lib.moe_last_error()
    assert gemm(N=1 << 20, K=1 << 13) == UNS
    assert gemm(S=1 << 31) == UNS and gemm(T=1 << 31) == UNS and gemm(S=-1) == INV
    assert gemm(rows=None) == INV and b"not S" in lib.moe_last_error()
    assert gemm(T=0) == INV and gemm(x=None) == INV and gemm(ws=None) == INV and gemm(off=None) == INV
    assert gemm(out=FAKE + 8) == INV and gemm(xs=FAKE + 2) == INV
    assert gemm(S=0, T=0, x=None) == B.MOE_OK


def test_other_calls_reject_the_new_flags():
    lib = B.load_library()
    for fl in (B.MOE_NORM_POST, B.MOE_NORM_PRE, B.MOE_GATE_CHANNEL, B.MOE_GATE_TOKEN, B.MOE_TRANSPOSED,
               B.MOE_GATED):
        assert lib.moe_route(FAKE, FAKE, None, 10, 128, 8, 2, fl, FAKE, FAKE, None, None) == INV
        assert lib.moe_combine(FAKE, None, FAKE, 10, 128, 2, fl, FAKE, None) == INV
        assert lib.moe_ffn_fwd(*([FAKE] * 6), 10, 128, 128, 8, 2, fl, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                               None) == INV


def test_python_refusals():
    """Shapes and types, checked before the library (host tensors: nothing is launched)."""
    bf, f32, u8, i32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32
    x = torch.zeros(4, 64, dtype=bf)
    q = mx.MX(torch.zeros(4, 32, dtype=u8), torch.zeros(4, 2, dtype=u8))
    w = mx.MX(torch.zeros(2, 64, 32, dtype=u8), torch.zeros(2, 64, 2, dtype=u8))
    off = torch.zeros(3, dtype=i32)
    with pytest.raises(ValueError, match="gate"):
        block.norm_forward(x, x, gate=torch.zeros(4, dtype=bf))
    with pytest.raises(ValueError, match="y: "):
        block.norm_forward(x, torch.zeros(3, 64, dtype=bf))
    with pytest.raises(ValueError, match="w_pre: dtype"):
        block.norm_forward(x, x, w_pre=torch.zeros(64, dtype=f32))
    with pytest.raises(ValueError, match="on the GPU"):
        block.norm_forward(x, x)
    with pytest.raises(ValueError, match="unsupported dtype"):
        block.norm_forward(x.half(), x.half())
    with pytest.raises(ValueError, match="neither dr nor dn"):
        block.norm_backward(None, None, x, x, None, None)
    with pytest.raises(ValueError, match="r: "):
        block.norm_backward(x, x, x, torch.zeros(5, 64, dtype=bf), None, None)
    with pytest.raises(ValueError, match="no blocks"):
        block.forward([], x)
    with pytest.raises(ValueError, match="no 4-bit experts"):
        block.infer([block.Block(w_pre=x[0], w_gate=x)], x)
    with pytest.raises(ValueError, match="multiple of 32"):
        mx.quantize(x[:, :48])
    with pytest.raises(ValueError, match="dimensions"):
        mx.quantize(x[0])
    with pytest.raises(ValueError, match="belong together"):
        mx.dequantize(mx.MX(q.codes, q.scales[:3]))
    with pytest.raises(ValueError, match="act 'gelu'"):
        mx.product(x, w, off, act="gelu")
    with pytest.raises(ValueError, match="w3 goes with"):
        mx.product(x, w, off, act="swiglu")
    with pytest.raises(ValueError, match="w3 goes with"):
        mx.product(x, w, off, w3=w, act="silu")
    with pytest.raises(ValueError, match="rows of 32"):
        mx.product(x[:, :32], w, off)
    with pytest.raises(ValueError, match="out: "):
        mx.product(x, w, off, out=torch.zeros(4, 32, dtype=bf))
    with pytest.raises(ValueError, match="offsets: 2 elements"):
        mx.product(q, w, off[:2])
    with pytest.raises(ValueError, match="neither"):
        mx.forward(x, x, None, mx.MXExperts(w, None, w), 1, False, rows="fp8")
    with pytest.raises(ValueError, match="do not fit"):
        mx.forward(torch.zeros(4, 128, dtype=bf), x, None, mx.MXExperts(w, None, w), 1, False)
    with pytest.raises(ValueError, match="on the GPU"):
        grads.clip([x], 1.0)
    with pytest.raises(TypeError, match="stream"):
        mx.quantize(x, stream=7)


# ---- the 64-bit forms ----------------------------------------------------------------------

@pytest.mark.parametrize("gate", [None, "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
def test_norm_gradient_formula_against_differences(gate, post, pre):
    """norm_bwd of block_ref against central differences of norm_fwd, in 64 bits: for the
    sum <dr, r> + <dn, n>, along a random direction of each input. Truncation of the
    difference is of order h^2 = 1e-8, rounding of order 2^-53 / h = 1e-12."""
    rng = np.random.default_rng(5)
    T, d, eps, scale, h = 5, 16, 1e-3, 0.7, 1e-4
    v = dict(res=rng.normal(size=(T, d)), y=rng.normal(size=(T, d)))
    shape = {None: None, "channel": (d,), "token": (T, 1), "full": (T, d)}[gate]
    if shape:
        v["gate"] = rng.normal(size=shape)
    if post:
        v["w_post"] = rng.normal(size=d)
    if pre:
        v["w_pre"] = rng.normal(size=d)
    dr, dn = rng.normal(size=(T, d)), rng.normal(size=(T, d))

    def fwd(q):
        return R.norm_fwd(q["res"], q["y"], q.get("gate"), q.get("w_post"), q.get("w_pre"), scale, eps)

    def loss(q):
        r, n, *_ = fwd(q)
        return (dr * r).sum() + ((dn * n).sum() if pre else 0.0)

    r, n, rpo, rpr, _ = fwd(v)
    g, _ = R.norm_bwd(dr, dn if pre else None, v["y"], r, rpo, rpr, v.get("gate"), v.get("w_post"),
                      v.get("w_pre"), scale)
    for name, gname in (("res", "dres"), ("y", "dy"), ("gate", "dgate"), ("w_post", "dw_post"), ("w_pre", "dw_pre")):
        if name not in v:
            continue
        u = rng.normal(size=v[name].shape)
        a = (loss({**v, name: v[name] + h * u}) - loss({**v, name: v[name] - h * u})) / (2 * h)
        assert abs(a - (g[gname] * u).sum()) < 1e-5, name


def test_mx_reference_values():
    """Hand-worked blocks: ties to the even code, saturation, the scale's floor."""
    x = np.zeros(32)
    x[:12] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -5.0, -0.25, 0.3]
    c, s = R.mx_quantize(x)
    assert s[0] == 127
    assert list(R.mx_values(c, s)[:12]) == [4, 0, 1, 1, 2, 2, 4, 4, 6, -4, 0, 0.5]
    assert np.signbit(R.mx_values(c, s)[10])
    c, s = R.mx_quantize(np.full(32, 2.0 ** -130))
    assert s[0] == 0 and (R.mx_values(c, s) == 0).all()        # 2^-3 of the smallest scale: a tie's lower side
    c, s = R.mx_quantize(np.full(32, 2.0 ** -128))
    assert s[0] == 0 and (R.mx_values(c, s) == 2.0 ** -128).all()
    for bad in (np.inf, -np.inf, np.nan):
        x[3] = bad
        assert R.mx_quantize(x)[1][0] == 255
    assert np.isnan(R.mx_values(*R.mx_quantize(x))).all()
