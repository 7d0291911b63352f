"""The gradient norm and clipping on the GPU against 64-bit sums. Bounds: the sum of n
squares is 64-bit (n 2^-53 relative), the norm is rounded once to float32; a clipped
value is a rounded coefficient times the value, rounded: two float32 half steps, and a
bfloat16 half step where it is stored so."""
import math

import numpy as np
import pytest
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import grads

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rand(n, dt, std=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + n)
    return (torch.randn(n, generator=g, device="cuda") * std).to(dt)


def _norm64(ts):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


def _lists():
    yield "one element", [_rand(1, F32)]
    yield "one small", [_rand(1000, BF)]
    yield "odd sizes", [_rand(n, dt) for n in (1, 3, 7, 8, 9, 255, 16383, 16385, 32769, 70001) for dt in (BF, F32)]
    yield "chunk borders", [_rand(n, F32) for n in (16384, 32768, 16384 * 3 - 1, 16384 * 3 + 1)]
    yield "unaligned views", [_rand(40001, F32)[1:], _rand(40001, BF)[1:], _rand(70003, BF)[3:-2], _rand(5, F32)[3:]]
    yield "empty ones", [_rand(0, F32), _rand(77, BF), _rand(0, BF), _rand(5000, F32)]
    yield "300 tensors", [_rand(100 + 37 * i, F32 if i % 3 else BF, seed=i) for i in range(300)]
    yield "many pieces", [_rand(50_000_001, F32), _rand(9_999_999, BF)]


@pytest.mark.parametrize("which", range(8))
def test_norm_and_clip(which):
    name, ts = list(_lists())[which]
    print(name, flush=True)
    ref = _norm64(ts)
    total, sumsq = grads.norm(ts)
    n = sum(t.numel() for t in ts)
    assert abs(float(sumsq) - ref * ref) <= (n + 4) * 2.0 ** -53 * 2 * ref * ref
    assert abs(float(total) - ref) <= ref * (2.0 ** -24 * 1.01)
    for max_norm in (ref / 3, ref * 2, 0.0, math.inf):
        c = min(1.0, max_norm / (ref + 1e-6))
        outs = [torch.full_like(t, 3.0) for t in ts]
        t2 = grads.clip(ts, max_norm, out=outs)
        assert torch.equal(t2, total)
        same = [t.clone() for t in ts]
        grads.clip(same, max_norm)
        for t, o, s in zip(ts, outs, same):
            assert torch.equal(o, s)
            if c == 1.0:
                assert torch.equal(o, t)
            v = t.double() * c
            half = 2.0 ** -24 if t.dtype == F32 else 2.0 ** -8
            assert bool(((o.double() - v).abs() <= v.abs() * (half + 2.0 ** -23) + 1e-40).all())


def test_values_that_float32_squares_lose():
    """1e25 squared is infinite in float32, 1e-30 squared zero: the 64-bit sum holds both."""
    for x in (1e25, 1e-30):
        t = torch.full((3000,), x, device="cuda")
        total, _ = grads.norm([t])
        ref = float(torch.tensor(x, dtype=F32)) * math.sqrt(3000)
        assert abs(float(total) - ref) <= ref * 2.0 ** -23


def test_infinite_and_nan_gradients():
    a, b = _rand(5000, F32), _rand(300, BF)
    for bad, c in ((math.nan, math.nan), (math.inf, 0.0)):
        a2 = a.clone()
        a2[4321] = bad
        out = [torch.empty_like(a2), torch.empty_like(b)]
        total = grads.clip([a2, b], 1.0, out=out)
        assert not math.isfinite(float(total))
        if math.isnan(c):
            assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all()
        else:
            assert torch.isnan(out[0][4321]) and (out[1] == 0).all() and int(torch.isnan(out[0]).sum()) == 1


def test_in_place_touches_only_its_elements():
    base = torch.full((40_010,), 5.0, device="cuda")
    view = base[5:40_003]
    grads.clip([view], 1.0)
    assert (base[:5] == 5).all() and (base[40_003:] == 5).all()
    assert abs(_norm64([view]) - 1.0) < 1e-5


def test_split_norms_add_up():
    """The squares of two halves' norms, added, clip as the whole does."""
    ts = [_rand(30_000, F32, seed=1), _rand(20_011, BF, seed=2), _rand(9, F32, seed=3)]
    whole = [t.clone() for t in ts]
    total = grads.clip(whole, 0.5)
    s = grads.norm(ts[:1])[1] + grads.norm(ts[1:])[1]
    parts = [t.clone() for t in ts]
    t1 = grads.clip(parts[:1], 0.5, sumsq=s)
    grads.clip(parts[1:], 0.5, sumsq=s)
    assert abs(float(t1) - float(total)) <= float(total) * 2.0 ** -23
    for a, b in zip(whole, parts):
        # two coefficients at most one float32 step apart: one more step of the stored type
        step = torch.finfo(a.dtype).eps
        assert bool(((a.double() - b.double()).abs() <= b.double().abs() * (step + 2.0 ** -23)).all())


def test_lists_dicts_none_and_nothing():
    t = _rand(100, F32)
    total, _ = grads.norm(dict(a=t, b=None))
    assert torch.equal(total, grads.norm([t])[0])
    u = _rand(33, BF)
    layers = [dict(dw1=t, dx=_rand(50, BF), d_gates=_rand(7, F32), dw3=None), dict(dX_slot=_rand(9, BF), dw1=u)]
    assert torch.equal(grads.norm(layers[0])[0], grads.norm([t])[0])
    assert torch.equal(grads.norm(layers)[0], grads.norm([t, u])[0])
    assert torch.equal(grads.norm([t, layers[1]])[0], grads.norm([t, u])[0])
    total, sumsq = grads.norm([])
    assert float(total) == 0.0 and float(sumsq) == 0.0
    assert float(grads.clip([None], 1.0)) == 0.0
    with pytest.raises(B.MoEError, match="overlap"):
        grads.clip([t, t], 1.0)
    with pytest.raises(B.MoEError, match="overlap"):
        grads.clip([t[:60], t[50:]], 1.0)
    out = torch.empty_like(t)
    with pytest.raises(B.MoEError, match="overlap"):
        grads.clip([t[:50], t[50:]], 1.0, out=[out[:50], out[10:60]])
    twice = [torch.empty_like(t), torch.empty_like(t)]
    grads.clip([t, t], 1e9, out=twice)            # read twice, written apart
    assert torch.equal(twice[0], t) and torch.equal(twice[1], t)
    with pytest.raises(ValueError, match="contiguous"):
        grads.norm([_rand(64, F32).view(8, 8).t()])
    with pytest.raises(ValueError, match="unsupported dtype"):
        grads.norm([t.half()])
    with pytest.raises(ValueError, match="outs"):
        grads.clip([t], 1.0, out=[out.bfloat16()])
    with pytest.raises(ValueError, match="out: 0"):
        grads.clip([t], 1.0, out=[])


def test_in_a_graph_and_on_another_stream():
    ts = [_rand(100_000, F32, seed=4), _rand(33_333, BF, seed=5)]
    outs = [torch.empty_like(t) for t in ts]
    graph = torch.cuda.CUDAGraph()
    grads.clip(ts, 1.0, out=outs)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        total = grads.clip(ts, 1.0, out=outs)
    for i in range(3):
        ts[0].mul_(1.7)
        want = [torch.empty_like(t) for t in ts]
        t2 = grads.clip(ts, 1.0, out=want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(total, t2) and all(torch.equal(a, b) for a, b in zip(outs, want)), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = grads.clip(ts, 1.0, out=outs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, t2) and all(torch.equal(a, b) for a, b in zip(outs, want))
