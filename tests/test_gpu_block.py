"""Stacks of residual blocks: forward and backward in float32 against 64-bit autograd on
the CPU, and a training step followed by 4-bit serving, as a program runs them."""
import numpy as np
import pytest
import torch

from paper_2601_05296_amd import block, grads, layer, mx
from tests.parity import TOL

pytestmark = pytest.mark.gpu


def _blocks(n, d, f, E, k, dt, post=True, gate=True, act="swiglu", scale=0.8, seed=0):
    g = torch.Generator().manual_seed(seed)

    def rnd(*s, std=1.0, mean=0.0):
        return (torch.randn(*s, generator=g) * std + mean).to(dt).cuda()

    return [block.Block(w_pre=rnd(d, std=0.1, mean=1.0), w_gate=rnd(E, d, std=0.2), w1=rnd(E, d, f, std=d ** -0.5),
                        w3=rnd(E, d, f, std=d ** -0.5) if act == "swiglu" else None,
                        w2=rnd(E, f, d, std=f ** -0.5), k=k, renorm=i % 2 == 0, act=act,
                        gate=rnd(d, std=0.2, mean=0.7) if gate else None,
                        w_post=rnd(d, std=0.1, mean=1.0) if post else None, res_scale=scale) for i in range(n)]


NAMES = ("w_pre", "w_gate", "w1", "w3", "w2", "gate", "w_post")
GRAD = dict(w_pre="dw_pre", w_gate="dw_gate", w1="dw1", w3="dw3", w2="dw2", gate="dgate", w_post="dw_post")


def _ref(blocks, x, ids, eps):
    """The stack in 64-bit torch on the CPU, with the experts that the GPU chose."""
    par = [{n: None if getattr(b, n) is None else getattr(b, n).double().cpu().requires_grad_() for n in NAMES}
           for b in blocks]
    x = x.double().cpu().requires_grad_()

    def rms(v, w):
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + eps) * w

    r = x
    for b, p, idx in zip(blocks, par, ids):
        n = rms(r, p["w_pre"])
        prob = torch.softmax(n @ p["w_gate"].t(), 1).gather(1, idx)
        if b.renorm:
            prob = prob / prob.sum(1, keepdim=True)
        a = torch.einsum("td,edf->tef", n, p["w1"])
        h = torch.relu(a) if b.act == "relu" else a * torch.sigmoid(a)
        if b.act == "swiglu":
            h = h * torch.einsum("td,edf->tef", n, p["w3"])
        O = torch.einsum("tef,efd->ted", h, p["w2"])
        y = (prob[:, :, None] * O.gather(1, idx[:, :, None].expand(-1, -1, O.shape[2]))).sum(1)
        if p["w_post"] is not None:
            y = rms(y, p["w_post"])
        r = b.res_scale * r + (y if p["gate"] is None else p["gate"] * y)
    return x, par, r


@pytest.mark.parametrize("post,gate,act", [(True, True, "swiglu"), (False, True, "silu"), (True, False, "relu"),
                                           (False, False, "swiglu")])
@pytest.mark.parametrize("n,T", [(1, 33), (3, 50)])
def test_stack_gradients(post, gate, act, n, T):
    blocks = _blocks(n, 128, 192, 4, 2, torch.float32, post, gate, act)
    x = torch.randn(T, 128, generator=torch.Generator().manual_seed(1)).cuda()
    dr = torch.randn(T, 128, generator=torch.Generator().manual_seed(2)).cuda()
    out, saved = block.forward(blocks, x, eps=1e-5)
    ids = [s.ids.long().cpu() for s in saved.layers]
    xr, par, want = _ref(blocks, x, ids, 1e-5)
    dx, g = block.backward(blocks, saved, dr)
    want.backward(dr.double().cpu())

    def close(name, a, b):
        e = float((a.double().cpu() - b).abs().max() / b.abs().max())
        assert e <= TOL["f32"], (name, e)

    close("out", out, want.detach())
    close("dx", dx, xr.grad)
    for i in range(n):
        for name in NAMES:
            if par[i][name] is None:
                assert g[i][GRAD[name]] is None
            else:
                close("%d %s" % (i, name), g[i][GRAD[name]], par[i][name].grad)


def test_stack_bf16_recompute_is_the_same():
    """The recompute policy of the layer under the stack: the stream bit for bit."""
    blocks = _blocks(2, 256, 256, 8, 2, torch.bfloat16)
    x = torch.randn(300, 256, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    a, s1 = block.forward(blocks, x)
    b, s2 = block.forward(blocks, x, recompute=True, chunk_tokens=100)
    assert torch.equal(a, b)
    dr = torch.ones_like(x)
    dx1, _ = block.backward(blocks, s1, dr)
    dx2, _ = block.backward(blocks, s2, dr)
    assert torch.equal(dx1, dx2)


@pytest.mark.parametrize("act", ["swiglu", "relu"])
def test_train_then_serve(act):
    """Forward, backward, clipping, a step, quantisation and 4-bit inference: the parts a
    training and serving program runs, in its order, each fed by the one before."""
    T, d, f, E, k = 200, 256, 320, 8, 2
    blocks = _blocks(2, d, f, E, k, torch.bfloat16, act=act)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    out, saved = block.forward(blocks, x)
    _, g = block.backward(blocks, saved, (out.float() * 0.01).bfloat16())
    flat = [t for b in g for n, t in b.items() if n != "d_gates" and t is not None]
    ref = sum(float((t.double() ** 2).sum()) for t in flat) ** 0.5
    total = grads.clip(flat, ref / 2)
    assert abs(float(total) - ref) <= ref * 2.0 ** -23
    after = sum(float((t.double() ** 2).sum()) for t in flat) ** 0.5
    assert abs(after - ref / 2) <= ref * 1e-5
    for b, gb in zip(blocks, g):
        for name in NAMES:
            p = getattr(b, name)
            if p is not None:
                setattr(b, name, (p.float() - 0.1 * gb[GRAD[name]].reshape(p.shape)).to(p.dtype))
        b.experts = mx.quantize_experts(b.w1, b.w3, b.w2)
    # served: the same as the trained path on the values that the codes stand for
    served = block.infer(blocks, x)
    dense = []
    for b in blocks:
        w = [None if t is None else mx.dequantize(t).transpose(1, 2).contiguous() for t in b.experts]
        dense.append(block.Block(b.w_pre, b.w_gate, *w, k=b.k, renorm=b.renorm, act=b.act, gate=b.gate,
                                 w_post=b.w_post, res_scale=b.res_scale))
    want, s = block.forward(dense, x)
    # a token near a tie of its router may choose otherwise after the first block's roundings
    far = (served.float() - want.float()).abs().amax(1) > 2e-2 * want.float().abs().max()
    assert int(far.sum()) <= 2, int(far.sum())
    four = block.infer(blocks, x, rows="mx")
    assert torch.isfinite(four.float()).all()
    one = block.infer(blocks, x[:1])
    assert (one.float() - served[:1].float()).abs().max() <= 2e-2 * want.float().abs().max()


def test_stack_on_another_stream_and_in_a_graph():
    blocks = _blocks(2, 256, 192, 8, 2, torch.bfloat16)
    for b in blocks:
        b.experts = mx.quantize_experts(b.w1, b.w3, b.w2)
    x = torch.randn(65, 256, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    dr = torch.ones_like(x)

    def step(stream=None):
        out, saved = block.forward(blocks, x, stream=stream)
        dx, g = block.backward(blocks, saved, dr, stream=stream)
        flat = [t for b in g for n, t in b.items() if n != "d_gates" and t is not None]
        total = grads.clip(flat, 0.5, stream=stream)
        return [out, dx, total, block.infer(blocks, x, stream=stream), *flat]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        x.mul_(1.1)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_two_streams_at_once():
    """The same calls side by side on two streams, with workspaces and results of their own."""
    g = torch.Generator(device="cuda").manual_seed(8)

    def rnd(*s):
        return torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)

    T, d, E, f = 3000, 1024, 8, 768
    w = [mx.quantize(rnd(E, f, d)) for _ in range(2)]
    off = torch.arange(E + 1, device="cuda", dtype=torch.int32) * (T // E)
    gate, wo, wr = rnd(d), rnd(d), rnd(d)
    ins = [[rnd(T, d) for _ in range(4)] for _ in range(2)]

    def calls(v):
        o = block.norm_forward(v[0], v[1], gate, wo, wr)
        b = block.norm_backward(v[2], v[3], v[1], o.r, o.rstd_post, o.rstd_pre, gate, wo, wr)
        h = mx.product(o.n, w[0], off, None, w[1], "swiglu")
        q = mx.product(mx.quantize(o.n), w[0], off)
        out = [torch.empty_like(t) for t in (b["dw_pre"], h)]
        n = grads.clip([b["dw_pre"], h], 0.5, out=out)
        return [o.r, o.n, b["dres"], b["dy"], b["dgate"], b["dw_post"], b["dw_pre"], h, q, n, *out]

    want = [calls(v) for v in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(calls(ins[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[i])), i
