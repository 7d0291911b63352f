"""Calls at the edges of what the operators around the layer take."""
import math

import numpy as np
import pytest
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import block, grads, layer, mx
from tests.test_gpu_mx import WIDE, _case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("act", ["none", "relu", "silu", "swiglu"])
@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("counts,N", [([1, 0, 1], 64), ([9, 2], 64), ([25, 30], 128), ([90, 40, 70, 80], WIDE)])
def test_product_keeps_nan_under_every_activation(act, x4, counts, N):
    """A NaN scale of one weight block, and a NaN row of x, in each core: NaN in that column
    of that expert and in that slot, whatever the activation, the formula's values elsewhere."""
    K, e = 192, len(counts) - 1
    dev, ref, tol = _case(counts, 20, K, N, act, x4, False, seed=2)
    dev["w"].scales[e, 6, 2] = 255
    if x4:
        dev["x"].scales[0, 1] = 255
    else:
        dev["x"][0, 7] = float("nan")
    out = mx.product(**dev).double().cpu().numpy()
    nan = np.zeros_like(ref, bool)
    nan[sum(counts) - counts[e]:, 6] = True
    nan[0] = True
    assert np.array_equal(np.isnan(out), nan)
    assert (np.abs(out - ref)[~nan] <= tol[~nan]).all()


@pytest.mark.parametrize("gate", [None, "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_norms_of_no_rows(gate, post, pre, dt):
    """An empty batch: empty tensors, and zeros for what is summed over the rows."""
    d = 64
    none, w = torch.empty(0, d, dtype=dt, device="cuda"), torch.ones(d, dtype=dt, device="cuda")
    g = {None: None, "channel": w, "token": none[:, :1].contiguous(), "full": none}[gate]
    o = block.norm_forward(none, none, g, w if post else None, w if pre else None)
    assert o.r.shape == (0, d)
    junk = [torch.full((d,), math.nan, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    b = block.norm_backward(none, none if pre else None, none, o.r, o.rstd_post, o.rstd_pre, g,
                            w if post else None, w if pre else None)
    assert b["dres"].shape == b["dy"].shape == (0, d)
    for k, on in (("dw_post", post), ("dw_pre", pre)):
        assert (b[k] is not None) == on and (not on or (b[k].shape == (d,) and not b[k].any()))
    if gate is not None:
        assert b["dgate"].shape == g.shape and not b["dgate"].any()


def test_clip_by_an_infinite_limit():
    """max_norm infinite leaves every gradient as it is, infinite ones among them; a NaN in the
    norm makes all NaN, also then."""
    a = torch.randn(5000, device="cuda")
    b = torch.randn(301, device="cuda").to(BF)
    a[4321], b[7] = math.inf, -math.inf
    for dst in (None, [torch.empty_like(a), torch.empty_like(b)]):
        g = [a.clone(), b.clone()]
        total = grads.clip(g, math.inf, out=dst)
        assert float(total) == math.inf
        assert torch.equal((dst or g)[0], a) and torch.equal((dst or g)[1], b)
    g = [a.clone(), b.clone()]
    g[0][1] = math.nan
    assert math.isnan(float(grads.clip(g, math.inf)))
    assert torch.isnan(g[0]).all() and torch.isnan(g[1]).all()


def _layer(T, dt=BF, act="swiglu"):
    g = torch.Generator(device="cuda").manual_seed(T)

    def rnd(*s):
        return (0.2 * torch.randn(*s, generator=g, device="cuda")).to(dt)

    return rnd(T, 64), rnd(4, 64), rnd(4, 64, 128), rnd(4, 64, 128) if act == "swiglu" else None, rnd(4, 128, 64)


def test_norm_of_all_that_a_backward_returns():
    """With keep=True the backward returns dX_slot and its sum over slots too: no parameters'."""
    x, wg, w1, w3, w2 = _layer(40)
    y, saved = layer.forward(x, wg, None, w1, w3, w2, 2, False, separate=True)
    g = layer.backward(saved, y, x, wg, w1, w3, w2, keep=True)
    par = [g[n] for n in ("dw1", "dw3", "dw2", "dw_gate")]
    assert torch.equal(grads.norm(g)[1], grads.norm(par)[1])
    before = {n: t.clone() for n, t in g.items()}
    grads.clip(g, 1e-3)
    for n, t in g.items():
        assert torch.equal(t, before[n]) == (n in ("dx", "dX_slot", "dx_ffn", "d_gates")), n


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("act", ["swiglu", "relu"])
@pytest.mark.parametrize("recompute", [False, True])
def test_stack_of_no_rows(dt, act, recompute):
    """A stack on an empty batch: an empty stream, and a zero gradient for every parameter."""
    bl = []
    for i in range(2):
        _, wg, w1, w3, w2 = _layer(i + 1, dt, act)
        one = torch.ones(64, dtype=dt, device="cuda")
        bl.append(block.Block(one, wg, w1, w3, w2, k=2, act=act, gate=one, w_post=one))
    x = torch.empty(0, 64, dtype=dt, device="cuda")
    y, saved = block.forward(bl, x, recompute=recompute)
    junk = [torch.full(s, math.nan, device="cuda") for s in ((4, 64, 128), (4, 64), (64,)) for _ in range(12)]
    torch.cuda.synchronize()
    del junk
    dx, g = block.backward(bl, saved, y)
    assert y.shape == dx.shape == (0, 64)
    for gb in g:
        assert {"dw1", "dw2", "dw_gate", "dgate", "dw_pre", "dw_post"} <= set(gb)
        for n, t in gb.items():
            assert t is None and n == "dw3" and act == "relu" or not t.any(), n
    assert float(grads.clip(g, 1.0)) == 0.0
    if dt == BF:
        for b in bl:
            b.experts = mx.quantize_experts(b.w1, b.w3, b.w2)
        for rows in ("bf16", "mx"):
            assert block.infer(bl, x, rows=rows).shape == (0, 64)


def test_layer_of_no_rows_returns_what_others_do():
    """The same keys, shapes and types as with tokens, whatever was asked to be kept."""
    for T in (3, 0):
        x, wg, w1, w3, w2 = _layer(3)
        x = x[:T].contiguous()
        y, saved = layer.forward(x, wg, None, w1, w3, w2, 2, False, separate=True)
        g = layer.backward(saved, y, x, wg, w1, w3, w2, keep=True)
        got = {n: (tuple(t.shape), t.dtype) for n, t in g.items()}
        if T:
            want = {n: ((0,) + s[1:] if s[0] in (3, 6) else s, dt) for n, (s, dt) in got.items()}
    assert list(got) == list(want) and got == want


def test_quantize_the_largest_width():
    """The widest transposed matrix that is taken, its last columns against the same alone."""
    R = (1 << 29) - 128
    x = torch.zeros(32, R, dtype=BF, device="cuda")
    tail = torch.randn(32, 10, generator=torch.Generator().manual_seed(0)).to(BF).cuda()
    x[:, -10:] = tail
    q, w = mx.quantize(x, True), mx.quantize(tail, True)
    assert torch.equal(q.codes[-10:], w.codes) and torch.equal(q.scales[-10:], w.scales)
    assert not q.codes[:-10].any() and not q.scales[:-10].any()


# rows of each expert, N: each core (few rows, 16 and 32 rows, tiles)
CORES = [([1, 0, 1], 64), ([9, 2], 64), ([25, 30], 128), ([90, 40, 70, 80], WIDE)]


@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("counts,N", CORES)
def test_product_ends_with_its_slots(x4, counts, N):
    """offsets that begin behind slot 0 (slots before are left as they were), and offsets that
    go on behind the S slots of the call: rows of the buffer behind them are."""
    K, S = 128, sum(counts)
    dev, ref, tol = _case(counts, 20, K, N, "none", x4, False, seed=5)
    x, xs = dev["x"] if x4 else (dev["x"], None)
    cut, off = S - counts[-1] // 2 - 1, dev["offsets"]
    slots = torch.arange(S, dtype=torch.int32, device="cuda")
    for rows, T in ((slots, S), (None, cut)):
        out = torch.full((S + 7, N), 77.0, dtype=BF, device="cuda")
        B.moe_mx_gemm(x, xs, *dev["w"], None, None, off, rows, T, cut, K, N, len(counts), 0, out)
        assert (out[cut:] == 77).all()
    e = len(counts) - 1
    w = [t[e:].contiguous() for t in dev["w"]]
    out = torch.full((S + 7, N), 77.0, dtype=BF, device="cuda")
    B.moe_mx_gemm(x, xs, *w, None, None, off[e:].clone(), None, S, S, K, N, 1, 0, out)
    got, lo = out.double().cpu().numpy(), S - counts[e]
    assert (np.abs(got[lo:S] - ref[lo:]) <= tol[lo:]).all() and (got[:lo] == 77).all() and (got[S:] == 77).all()


@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("counts,N", CORES)
def test_product_of_offsets_that_are_none(x4, counts, N):
    """Negative, decreasing and huge offsets: nothing outside the result's rows is written."""
    K, S, E = 64, sum(counts), len(counts)
    dev, *_ = _case(counts, 20, K, N, "none", x4, False, seed=6)
    x, xs = dev["x"] if x4 else (dev["x"], None)
    buf = torch.full((S + 128, N), 77.0, dtype=BF, device="cuda")
    big = (1 << 31) - 1
    for off in ([0] + [big] * E, [-1 - big] * E + [big], [S] + [0] * E, [-5] * E + [S], [big] * E + [0],
                [S + 50] * E + [S + 90], [big - 3] * E + [big], [0, S, -S, big][:E] + [S] * (E + 1 - len([0, S, -S, big][:E]))):
        print(off, flush=True)
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        B.moe_mx_gemm(x, xs, *dev["w"], None, None, off, None, S, S, K, N, E, 0, buf[64:64 + S])
        torch.cuda.synchronize()
        assert (buf[:64] == 77).all() and (buf[64 + S:] == 77).all()


def test_product_beside_its_inputs():
    """Results right behind x in one buffer are taken, over x they are refused."""
    K = N = 128
    S = 40
    dev, ref, tol = _case([S], 20, K, N, "none", False, False, seed=7)
    buf = torch.zeros(2 * S, K, dtype=BF, device="cuda")
    buf[:S] = dev["x"]
    dev["x"] = buf[:S]
    for out in (buf[:S], buf[S - 1:2 * S - 1]):
        with pytest.raises(B.MoEError, match="out overlaps x"):
            mx.product(**dev, out=out)
    mx.product(**dev, out=buf[S:])
    assert (np.abs(buf[S:].double().cpu().numpy() - ref) <= tol).all()


def test_calls_of_the_binding_are_those_of_the_modules():
    """One function of the binding for each entry point, on the caller's own buffers."""
    ts = [torch.randn(1000, device="cuda"), torch.randn(77, device="cuda").to(BF)]
    tl = B.TensorList(ts)
    norm, sumsq = torch.empty((), device="cuda"), torch.empty((), dtype=torch.float64, device="cuda")
    n = B.moe_grad_norm_workspace_size(tl.n)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.moe_grad_norm(tl, sumsq, norm, ws, n)
    want = grads.norm(ts)
    assert torch.equal(norm, want[0]) and torch.equal(sumsq, want[1])
    q = mx.quantize(ts[0][:960].reshape(10, 96))
    for dt, fl in ((BF, B.MOE_BF16), (F32, B.MOE_F32)):
        out = torch.empty(10, 96, dtype=dt, device="cuda")
        B.moe_mx_dequantize(q.codes, q.scales, 10, 96, fl, out)
        assert torch.equal(out, mx.dequantize(q, dt))
    with pytest.raises(ValueError, match="workspace"):
        B.moe_grad_norm(tl, sumsq, norm, ws[:8], n)
    with pytest.raises(ValueError, match="sumsq: dtype"):
        B.moe_grad_norm(tl, norm, norm, ws, n)
    with pytest.raises(ValueError, match="out: dtype"):
        B.moe_mx_dequantize(q.codes, q.scales, 10, 96, B.MOE_F32, torch.empty(960, dtype=BF, device="cuda"))
    with pytest.raises(ValueError, match="scales: 20 elements"):
        B.moe_mx_dequantize(q.codes, q.scales[:, :2].contiguous(), 10, 96, B.MOE_BF16, out)
