"""The block norms, clipping and the 4-bit operators where places in a tensor pass 32 bits:
most of each tensor is zeros, its last rows are compared with the same rows alone."""
import math

import pytest
import torch

from paper_2601_05296_amd import block, grads, mx

pytestmark = pytest.mark.gpu
BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def _rand(*s, seed=0, dt=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*s, generator=g, device="cuda").to(dt)


def test_norms():
    T, d, m = 300_001, 8192, 5
    res, y, dr, dn = (torch.zeros(T, d, dtype=BF, device="cuda") for _ in range(4))
    tails = [_rand(m, d, seed=i) for i in range(4)]
    for t, v in zip((res, y, dr, dn), tails):
        t[-m:] = v
    gate, wo, wr = _rand(d, seed=5), _rand(d, seed=6), _rand(d, seed=7)
    o = block.norm_forward(res, y, gate, wo, wr, 0.7)
    w = block.norm_forward(tails[0], tails[1], gate, wo, wr, 0.7)
    assert torch.equal(o.r[-m:], w.r) and torch.equal(o.n[-m:], w.n)
    assert torch.equal(o.rstd_post[-m:], w.rstd_post) and torch.equal(o.rstd_pre[-m:], w.rstd_pre)
    assert not o.r[:-m].any() and not o.n[:-m].any()
    g = block.norm_backward(dr, dn, y, o.r, o.rstd_post, o.rstd_pre, gate, wo, wr, 0.7)
    v = block.norm_backward(tails[2], tails[3], tails[1], w.r, w.rstd_post, w.rstd_pre, gate, wo, wr, 0.7)
    assert torch.equal(g["dres"][-m:], v["dres"]) and torch.equal(g["dy"][-m:], v["dy"])
    assert not g["dres"][:-m].any() and not g["dy"][:-m].any()
    for k in ("dgate", "dw_post", "dw_pre"):   # five terms, added in another order
        assert torch.allclose(g[k], v[k], rtol=0, atol=8 * 2.0 ** -24 * 5 * float(v[k].abs().max() + 100)), k


def test_clip():
    n, m = (1 << 31) + 12345, 1000
    g = torch.zeros(n, dtype=F32, device="cuda")
    tail = _rand(m, dt=F32)
    g[-m:] = tail
    want = math.sqrt(float((tail.double() ** 2).sum()))
    out = torch.full((n,), 7.0, dtype=F32, device="cuda")
    norm = grads.clip([g], 1.0, out=[out])
    assert abs(float(norm) - want) <= want * 2.0 ** -23
    assert not out[:-m].any()
    c = torch.tensor(1.0 / (want + 1e-6), dtype=torch.float64).float().cuda()
    assert torch.equal(out[-m:], tail * c)


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize(transpose):
    R, K, m = (1 << 26) + 66, 96, 10
    shape = (K, R) if transpose else (R, K)
    x = torch.zeros(*shape, dtype=BF, device="cuda")
    tail = _rand(m, K)
    if transpose:
        x[:, -m:] = tail.t()
    else:
        x[-m:] = tail
    q, w = mx.quantize(x, transpose), mx.quantize(tail)
    assert torch.equal(q.codes[-m:], w.codes) and torch.equal(q.scales[-m:], w.scales)
    assert not q.codes[:-m].any() and not q.scales[:-m].any()
    del x
    v = mx.dequantize(q)
    assert torch.equal(v[-m:], mx.dequantize(w)) and not v[:-m].any()


@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("S", [40, 3000])
def test_product_far_rows(x4, S):
    """Rows of x, and results, beyond 4 GB."""
    K, N, m = 8192, 11328, 64
    T = 1_200_000 if x4 else 300_000
    tail = _rand(m, K)
    w = mx.quantize(_rand(2, N, K, seed=2))
    if x4:
        small = mx.quantize(tail)
        x = mx.MX(torch.zeros(T, K // 2, dtype=U8, device="cuda"), torch.full((T, K // 32), 127, dtype=U8, device="cuda"))
        x.codes[-m:], x.scales[-m:] = small
    else:
        small, x = tail, torch.zeros(T, K, dtype=BF, device="cuda")
        x[-m:] = tail
    rows = torch.randint(0, m, (S,), dtype=torch.int32, generator=torch.Generator().manual_seed(S)).cuda()
    off = torch.tensor([0, S // 3, S], dtype=torch.int32, device="cuda")
    got = mx.product(x, w, off, rows + (T - m))
    assert torch.equal(got, mx.product(small, w, off, rows)) and got.abs().sum() > 0


def test_product_far_results():
    K, N, S, m = 64, 14336, 160_000, 300
    w = mx.quantize(_rand(1, N, K, seed=2))
    x = torch.zeros(S, K, dtype=BF, device="cuda")
    x[-m:] = _rand(m, K)
    got = mx.product(x, w, torch.tensor([0, S], dtype=torch.int32, device="cuda"))
    want = x[-m:].double() @ mx.dequantize(w, F32)[0].double().t()
    mag = x[-m:].double().abs() @ mx.dequantize(w, F32)[0].double().abs().t()
    assert not got[:-m].any()
    assert bool(((got[-m:].double() - want).abs() <= want.abs() * 2.0 ** -8 * 1.01 + (K + 16) * 2.0 ** -24 * mag).all())
