"""The block norms on the GPU against their 64-bit forms (block_ref), forward and
backward. Bounds: an output is rounded once (HALF of its value); its float32 terms pass
through at most 16 elementwise roundings and a sum of at most 16 values a lane, 6 lane
steps and 8 waves, so 64 float32 half steps of the terms' magnitude cover it; a column
sum adds at most T + 64 more."""
import numpy as np
import pytest
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import block
from tests import block_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _make(T, d, dtype, gate, post, pre, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]

    def rnd(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g) * std + mean).to(dt)

    v = dict(res=rnd(T, d, std=2.0), y=rnd(T, d), dr=rnd(T, d), gate=None, w_post=None, w_pre=None, dn=None)
    if gate:
        v["gate"] = rnd(*{"channel": (d,), "token": (T, 1), "full": (T, d)}[gate], std=0.5, mean=0.3)
    if post:
        v["w_post"] = rnd(d, std=0.2, mean=1.0)
    if pre:
        v["w_pre"], v["dn"] = rnd(d, std=0.2, mean=1.0), rnd(T, d)
    return v


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _close(name, got, ref, mag, half, c):
    got = _np(got)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    tol = half * np.abs(ref) * (1 + 2.0 ** -7) + c * R.U32 * mag + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), float(np.max(np.abs(got - ref) / tol)))


def _check(v, dtype, scale, T, d):
    n = {k: _np(t) for k, t in v.items()}
    dev = {k: None if t is None else t.cuda() for k, t in v.items()}
    half = R.HALF[dtype]
    o = block.norm_forward(dev["res"], dev["y"], dev["gate"], dev["w_post"], dev["w_pre"], scale, EPS)
    r, nn, rpo, rpr, mag = R.norm_fwd(n["res"], n["y"], n["gate"], n["w_post"], n["w_pre"], scale, EPS)
    _close("r", o.r, r, mag, half, 64)
    if rpo is not None:
        _close("rstd_post", o.rstd_post, rpo, rpo, R.U32, 64)
    if rpr is not None:
        # r's error enters as it is: relative to the row's own size
        rel = np.sqrt((mag ** 2).mean(1) / ((r ** 2).mean(1) + EPS))
        _close("rstd_pre", o.rstd_pre, rpr, rpr * (1 + rel), R.U32, 64)
        k = rpr[:, None] * np.abs(n["w_pre"])
        _close("n", o.n, nn, k * mag + np.abs(nn) * (1 + rel[:, None]), half, 64)
    # the backward on the forward's own outputs, taken as given
    g = block.norm_backward(dev["dr"], dev["dn"], dev["y"], o.r, o.rstd_post, o.rstd_pre, dev["gate"],
                            dev["w_post"], dev["w_pre"], scale)
    ref, m = R.norm_bwd(n["dr"], n["dn"], n["y"], _np(o.r), _np(o.rstd_post), _np(o.rstd_pre), n["gate"],
                        n["w_post"], n["w_pre"], scale)
    assert {k for k, t in g.items() if t is not None} == set(ref)
    for k in ref:
        summed = k in ("dw_pre", "dw_post") or k == "dgate" and n["gate"].shape != n["y"].shape
        _close(k, g[k], ref[k], m[k], R.U32 if summed else half, 64 + (T if summed and ref[k].ndim == 1 else d // 64))


@pytest.mark.parametrize("T,d,dtype", [
    (1, 8, "bf16"), (3, 64, "bf16"), (2, 520, "bf16"), (130, 512, "bf16"), (67, 1024, "bf16"),
    (5, 2048, "bf16"), (9, 2056, "bf16"), (1021, 2880, "bf16"), (33, 4096, "bf16"), (17, 8192, "bf16"),
    (1, 8, "f32"), (19, 256, "f32"), (7, 264, "f32"), (70, 1000, "f32"), (11, 2048, "f32"),
    (513, 2880, "f32"), (6, 4104, "f32"), (13, 8192, "f32"),
])
def test_norms_over_widths(T, d, dtype):
    """Every shape of the row kernels, ragged rows, all three parts on."""
    print(T, d, dtype, flush=True)
    _check(_make(T, d, dtype, "channel", True, True, T + d), dtype, 0.7, T, d)


@pytest.mark.parametrize("gate", [None, "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_over_variants(gate, post, pre, dtype):
    for T, d in ((37, 256), (6, 2304), (21, 1024), (300, 3080)):
        print(T, d, flush=True)
        _check(_make(T, d, dtype, gate, post, pre, 3), dtype, 1.0, T, d)


@pytest.mark.parametrize("T,d", [(9001, 64), (6007, 1536), (3001, 4096), (5003, 1000), (2999, 3048), (1500, 8000)])
def test_norms_many_rows_a_workgroup(T, d):
    print(T, d, flush=True)
    _check(_make(T, d, "bf16", "token", True, True, 1), "bf16", 0.5, T, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_without_a_block_output(dtype):
    """The first norm of a stack: n of res alone, and its gradient with and without dr."""
    T, d = 35, 768
    v = _make(T, d, dtype, None, False, True, 4)
    n = {k: _np(t) for k, t in v.items()}
    dev = {k: None if t is None else t.cuda() for k, t in v.items()}
    o = block.norm_forward(dev["res"], w_pre=dev["w_pre"], eps=EPS)
    assert o.r is None and o.rstd_post is None
    r, nn, _, rpr, mag = R.norm_fwd(n["res"], None, None, None, n["w_pre"], 1.0, EPS)
    _close("n", o.n, nn, np.abs(nn) * 2, R.HALF[dtype], 64)
    for dr in (dev["dr"], None):
        g = block.norm_backward(dr, dev["dn"], None, dev["res"], None, o.rstd_pre, w_pre=dev["w_pre"], block=False)
        ref, m = R.norm_bwd(n["dr"] if dr is not None else None, n["dn"], None, n["res"], None, _np(o.rstd_pre),
                            None, None, n["w_pre"], 1.0)
        assert g["dy"] is None and g["dgate"] is None
        _close("dres", g["dres"], ref["dres"], m["dres"], R.HALF[dtype], 64)
        _close("dw_pre", g["dw_pre"], ref["dw_pre"], m["dw_pre"], R.U32, 64 + T)


def test_norm_rows_of_zeros_large_values_and_nan():
    """A row of zeros keeps finite outputs, a NaN or infinite row does not reach the others,
    and values far from one keep their precision."""
    T, d = 9, 640
    v = _make(T, d, "f32", "channel", True, True, 8)
    v["y"][2] = 0.0
    v["res"][2] = 0.0
    v["y"][4] *= 1e15
    v["res"][5] *= 1e-12
    _check(v, "f32", 1.0, T, d)
    w = {k: None if t is None else t.cuda() for k, t in v.items()}
    base = block.norm_forward(w["res"], w["y"], w["gate"], w["w_post"], w["w_pre"])
    for row, bad in ((0, float("nan")), (8, float("inf"))):
        y = w["y"].clone()
        y[row, 3] = bad
        o = block.norm_forward(w["res"], y, w["gate"], w["w_post"], w["w_pre"])
        others = [i for i in range(T) if i != row]
        assert torch.equal(o.n[others], base.n[others]) and torch.equal(o.r[others], base.r[others])
        assert not torch.isfinite(o.r[row]).all()


def test_norm_in_place_and_repeatable():
    """r over res, n over y; dres and dy over dr and dn: the bits of separate outputs."""
    T, d = 3000, 2048
    v = {k: None if t is None else t.cuda() for k, t in _make(T, d, "bf16", "channel", True, True, 6).items()}
    f32 = dict(dtype=torch.float32, device="cuda")
    fl = B.MOE_NORM_POST | B.MOE_NORM_PRE | B.MOE_GATE_CHANNEL
    o = block.norm_forward(v["res"], v["y"], v["gate"], v["w_post"], v["w_pre"])
    a, b = v["res"].clone(), v["y"].clone()
    po, pr = torch.empty(T, **f32), torch.empty(T, **f32)
    B.moe_norm_fwd(a, b, v["gate"], v["w_post"], v["w_pre"], 1.0, EPS, T, d, fl, a, b, po, pr)
    assert torch.equal(a, o.r) and torch.equal(b, o.n) and torch.equal(po, o.rstd_post) and torch.equal(pr, o.rstd_pre)
    args = (v["dr"], v["dn"], v["y"], o.r, o.rstd_post, o.rstd_pre, v["gate"], v["w_post"], v["w_pre"])
    g = block.norm_backward(*args)
    again = block.norm_backward(*args)
    assert all(torch.equal(g[k], again[k]) for k in g)
    dr, dn = v["dr"].clone(), v["dn"].clone()
    dg, dwo, dwr = (torch.empty(d, **f32) for _ in range(3))
    wsb = B.moe_norm_bwd_workspace_size(T, d, fl)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    B.moe_norm_bwd(dr, dn, v["y"], o.r, v["gate"], v["w_post"], v["w_pre"], po, pr, 1.0, T, d, fl, dr, dn, dg,
                   dwo, dwr, ws, wsb)
    assert torch.equal(dr, g["dres"]) and torch.equal(dn, g["dy"]) and torch.equal(dg, g["dgate"])
    assert torch.equal(dwo, g["dw_post"]) and torch.equal(dwr, g["dw_pre"])


def test_norm_writes_its_rows_only():
    """Rows behind T, and without rows everything but the zeroed sums, are left as they were."""
    T, d = 21, 1032
    v = {k: None if t is None else t.cuda() for k, t in _make(T + 4, d, "bf16", None, True, True, 2).items()}
    r, n = torch.full_like(v["res"], 7.0), torch.full_like(v["res"], 7.0)
    fl = B.MOE_NORM_POST | B.MOE_NORM_PRE
    B.moe_norm_fwd(v["res"], v["y"], None, v["w_post"], v["w_pre"], 1.0, EPS, T, d, fl, r, n)
    assert (r[T:] == 7).all() and (n[T:] == 7).all() and not (r[:T] == 7).all()
    none = torch.empty(0, d, dtype=torch.bfloat16, device="cuda")
    o = block.norm_forward(none, none, None, v["w_post"], v["w_pre"])
    assert o.r.shape == (0, d) and o.n.shape == (0, d)
    g = block.norm_backward(none, none, none, o.r, o.rstd_post, o.rstd_pre, w_post=v["w_post"], w_pre=v["w_pre"])
    assert g["dres"].shape == (0, d) and (g["dw_post"] == 0).all() and (g["dw_pre"] == 0).all()


def test_norm_on_another_stream_and_in_a_graph():
    T, d = 257, 2048
    v = {k: None if t is None else t.cuda() for k, t in _make(T, d, "bf16", "token", True, True, 5).items()}

    def step(stream=None):
        o = block.norm_forward(v["res"], v["y"], v["gate"], v["w_post"], v["w_pre"], stream=stream)
        g = block.norm_backward(v["dr"], v["dn"], v["y"], o.r, o.rstd_post, o.rstd_pre, v["gate"], v["w_post"],
                                v["w_pre"], stream=stream)
        return [o.r, o.n, *g.values()]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        v["y"].mul_(1.5)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
