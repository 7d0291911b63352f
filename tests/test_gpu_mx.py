"""Microscaled 4-bit values and the grouped products over them, on the GPU.

Quantisation is held to the definition bit for bit. A product's float32 sum of K terms is
off by at most (K + 16) half steps of the terms' magnitudes, an activation adds its own
few, and the result is rounded once to bfloat16."""
import numpy as np
import pytest
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import layer, mx
from tests import block_ref as R
from tests.parity import launched

pytestmark = pytest.mark.gpu
BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def _check_quant(x, transpose=False):
    """x (CPU): codes, scales and values against the 64-bit form. NaN blocks: scale alone."""
    q = mx.quantize(x.cuda(), transpose)
    v = x.double().numpy()
    v = np.ascontiguousarray(np.swapaxes(v, -1, -2)) if transpose else v
    with np.errstate(invalid="ignore"):
        codes, scales = R.mx_quantize(v)
    got_c, got_s = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    assert np.array_equal(got_s, scales)
    ok = np.repeat(scales != 255, 16, -1)
    assert np.array_equal(got_c[ok], codes[ok])
    for dt in (BF, F32):
        got = mx.dequantize(q, dt).double().cpu().numpy()
        want = R.mx_values(got_c, scales)
        assert np.array_equal(got, want, equal_nan=True), dt


def test_quantize_every_bfloat16():
    """Every bfloat16 pattern, each beside 31 others of its own size (so that every one is
    rounded under a scale near its own), and under a scale set by a value 8 times its size."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    x = bits.view(BF).reshape(-1, 32)
    _check_quant(x)
    _check_quant(x.reshape(64, -1, 32).transpose(0, 1).reshape(-1, 32 * 64).contiguous())
    y = x.clone().float()
    finite = torch.isfinite(y) & (y.abs() < 2.0 ** 120)
    y = torch.where(finite, y, torch.zeros(()))
    y[:, 0] = y.abs().amax(1) * 8
    _check_quant(y.to(BF))
    _check_quant(y)


def test_quantize_float32_around_the_borders():
    """float32 values one step on either side of each rounding border, under every scale."""
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    near = torch.cat([mids, torch.nextafter(mids, mids + 1), torch.nextafter(mids, mids - 1), mids / 3])
    near = torch.cat([torch.tensor([4.0]), near[:31]])
    assert near.numel() == 32
    e = torch.arange(-126, 123, dtype=torch.float64)
    x = (near.double()[None] * torch.pow(2.0, e)[:, None])
    x = torch.cat([x, -x], 1).float()
    _check_quant(x)
    assert torch.isfinite(x).all()


@pytest.mark.parametrize("shape", [(1, 32), (3, 96), (7, 11, 64), (1, 8192), (2049, 160), (5, 2, 3, 32)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_quantize_rows(shape, dt):
    g = torch.Generator().manual_seed(sum(shape))
    x = torch.randn(*shape, generator=g) * torch.exp(torch.randn(*shape, generator=g) * 3)
    x.view(-1, 32)[0] = 0.0
    x.view(-1)[-1] = float("inf")
    _check_quant(x.to(dt))


@pytest.mark.parametrize("shape", [(32, 2), (64, 130), (3, 96, 62), (2, 288, 128), (5, 2880, 64), (1, 8192, 6)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_quantize_transposed(shape, dt):
    g = torch.Generator().manual_seed(sum(shape))
    x = torch.randn(*shape, generator=g) * torch.exp(torch.randn(*shape, generator=g))
    x[..., 5, 1] = float("nan")
    _check_quant(x.to(dt), transpose=True)


def test_dequantize_every_code_and_scale():
    scales = torch.arange(256, dtype=U8).reshape(256, 1)
    codes = torch.arange(16, dtype=U8)
    codes = (codes | (15 - codes) << 4).repeat(256, 1)
    q = mx.MX(codes.cuda(), scales.cuda())
    want = R.mx_values(codes.numpy(), scales.numpy())
    for dt in (BF, F32):
        got = mx.dequantize(q, dt).double().cpu().numpy()
        with np.errstate(over="ignore"):
            w = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
        assert np.array_equal(got, w, equal_nan=True)


def test_quantize_leaves_what_is_behind():
    x = torch.randn(3, 64).cuda()
    codes, scales = torch.full((200,), 9, dtype=U8).cuda(), torch.full((40,), 9, dtype=U8).cuda()
    B.moe_mx_quantize(x, 1, 3, 64, B.MOE_F32, codes, scales)
    assert (codes[96:] == 9).all() and (scales[6:] == 9).all()
    assert mx.quantize(x[:0]).codes.shape == (0, 32)
    assert mx.dequantize(mx.quantize(x[:0])).shape == (0, 64)


# ---- grouped products ----------------------------------------------------------------------

def _experts(gen, E, N, K):
    """Codes of every kind, scales of a few powers of two around 2^-4."""
    codes = torch.randint(0, 256, (E, N, K // 2), generator=gen, dtype=torch.int32).to(U8)
    scales = torch.randint(120, 126, (E, N, K // 32), generator=gen, dtype=torch.int32).to(U8)
    return mx.MX(codes, scales)


def _case(counts, T, K, N, act, x4, gather, seed=0, spare=0):
    """counts: rows of each expert. Returns the device arguments and the 64-bit result with
    its bound; ``spare`` slots lie behind offsets[E]."""
    gen = torch.Generator().manual_seed(seed)
    E, S = len(counts), sum(counts) + spare
    off = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32)
    rows = torch.randint(0, T, (S,), generator=gen, dtype=torch.int32) if gather else None
    n = T if gather else S
    x = (torch.randn(n, K, generator=gen) * torch.exp(torch.randn(n, 1, generator=gen))).to(BF)
    xq = None
    if x4:
        codes, scales = R.mx_quantize(x.double().numpy())
        xq = mx.MX(torch.from_numpy(codes), torch.from_numpy(scales))
        xv = R.mx_values(codes, scales)
    else:
        xv = x.double().numpy()
    w = _experts(gen, E, N, K)
    w3 = _experts(gen, E, N, K) if act == "swiglu" else None
    if gather:
        xv = xv[rows.numpy()]
    ref, tol = np.zeros((S - spare, N)), np.zeros((S - spare, N))
    u = (K + 16) * R.U32
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        if lo == hi:
            continue
        v = R.mx_values(w.codes[e].numpy(), w.scales[e].numpy()).T
        a, ea = xv[lo:hi] @ v, u * (np.abs(xv[lo:hi]) @ np.abs(v))
        if act == "relu":
            a = np.maximum(a, 0.0)
        elif act in ("silu", "swiglu"):
            with np.errstate(over="ignore"):
                sg = 1.0 / (1.0 + np.exp(-a))
            # exp(-a) is off by about |a| + 8 half steps, SiLU's slope is at most 1.1
            h, eh = a * sg, 1.1 * ea + np.abs(a * sg) * (2 * np.abs(a) + 16) * R.U32
            if act == "swiglu":
                v3 = R.mx_values(w3.codes[e].numpy(), w3.scales[e].numpy()).T
                b, eb = xv[lo:hi] @ v3, u * (np.abs(xv[lo:hi]) @ np.abs(v3))
                h, eh = h * b, eh * (np.abs(b) + eb) + (np.abs(h) + eh) * eb
            a, ea = h, eh
        ref[lo:hi], tol[lo:hi] = a, ea
    tol = tol * 1.01 + np.abs(ref) * 2.0 ** -8 * 1.01 + 1e-30
    dev = dict(x=mx.MX(*(t.cuda() for t in xq)) if x4 else x.cuda(), w=mx.MX(*(t.cuda() for t in w)),
               offsets=off.cuda(), rows=None if rows is None else rows.cuda(),
               w3=None if w3 is None else mx.MX(*(t.cuda() for t in w3)), act=act)
    return dev, ref, tol


def _run(dev, ref, tol, spare=0):
    S = ref.shape[0] + spare
    out = torch.full((S, ref.shape[1]), 77.0, dtype=BF, device="cuda")
    mx.product(**dev, out=out)
    got = out.double().cpu().numpy()
    bad = ~(np.abs(got[:ref.shape[0]] - ref) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], float(np.max(np.abs(got[:ref.shape[0]] - ref) / tol)))
    assert (got[ref.shape[0]:] == 77.0).all()


# rows of each expert, chosen so that the mean picks each core where N is WIDE: streams of 4,
# 16 and 32 rows, tiles of 64, 128 and 256 (narrow products leave CUs idle: streams)
WIDE = 11328   # 177 x 64
LOADS = {
    "one": [0, 0, 1, 0], "same": [0, 7, 0, 0, 0, 0, 0, 0], "few": [3, 0, 17, 1, 0, 16, 0], "some": [40, 2, 0, 33, 16],
    "tile64": [64, 1, 0, 130, 33], "tile128": [129, 128, 3, 0, 200], "tile256": [256, 300, 0, 1, 700, 255],
}


@pytest.mark.parametrize("load", LOADS)
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("x4", [False, True])
def test_product_over_loads(load, act, x4):
    counts = LOADS[load]
    for K, N, gather in ((320, 192, True), (64, 64, False), (576, 320, False)):
        spare = 3 if gather else 0
        print(load, act, x4, K, N, gather, flush=True)
        dev, ref, tol = _case(counts, 50, K, N, act, x4, gather, seed=K + N, spare=spare)
        _run(dev, ref, tol, spare)


def test_product_loads_reach_every_core():
    names = {}
    for load, counts in LOADS.items():
        dev, *_ = _case(counts, 50, 128, WIDE, "none", False, True)
        names[load] = launched(lambda: mx.product(**dev))
    assert [names[n] for n in LOADS] == [["mx_stream"]] * 4 + [["mx_tile"]] * 3


@pytest.mark.parametrize("load", ["some", "tile64", "tile128", "tile256"])
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("x4", [False, True])
def test_product_wide_loads(load, act, x4):
    """Tiles, over depths of one slice, of slices cut short and of rows that are no whole slices."""
    for K, gather in ((64, True), (320, False), (576, True), (1024, False)) + (() if act == "swiglu" else ((4160, True),)):
        print(load, act, x4, K, gather, flush=True)
        dev, ref, tol = _case(LOADS[load], 50, K, WIDE, act, x4, gather, seed=K, spare=3)
        _run(dev, ref, tol, 3)


@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("load", ["few", "tile128"])
def test_product_activations(load, act):
    _run(*_case(LOADS[load], 40, 256, 128, act, False, True, seed=9))
    _run(*_case(LOADS[load], 40, 128, WIDE, act, True, True, seed=10))


@pytest.mark.parametrize("K,N", [(64, 128), (128, 64), (192, 256), (1408, 2048), (2880, 2880), (4096, 192), (8192, 64)])
@pytest.mark.parametrize("x4", [False, True])
def test_product_widths(K, N, x4):
    """Depths that end inside a slice or a wave's share of K, widths that end inside a tile."""
    for counts in ([5, 0, 9], [70, 31]):
        print(K, N, x4, counts, flush=True)
        _run(*_case(counts, 33, K, N, "swiglu", x4, True, seed=1))


@pytest.mark.parametrize("K", [4096, 4160, 8256, 14336])
@pytest.mark.parametrize("x4", [False, True])
def test_product_deep(K, x4):
    """Long sums on few workgroups, the scales reloaded on the way, rows not whole slices."""
    for counts in ([1, 0, 1], [11, 0, 2], [25, 9], [90, 41], [300]):
        print(K, x4, counts, flush=True)
        _run(*_case(counts, 27, K, 64, "none", x4, len(counts) > 1, seed=K))


@pytest.mark.parametrize("x4", [False, True])
def test_product_wide(x4):
    """More workgroups than CUs for a row or two, and wide enough for every column split."""
    for counts in ([1, 0, 2, 0, 1, 0], [20, 30]):
        _run(*_case(counts, 5, 192, 14336, "swiglu", x4, True, seed=7))


@pytest.mark.parametrize("x4", [False, True])
def test_product_many_experts(x4):
    rng = np.random.default_rng(3)
    for E, mean in ((256, 0.4), (256, 6), (130, 40)):
        counts = rng.poisson(mean, E).tolist()
        print(E, mean, sum(counts), flush=True)
        _run(*_case(counts, 64, 64, 64, "none", x4, True, seed=E))


@pytest.mark.parametrize("x4", [False, True])
def test_product_many_experts_whole_rounds(x4):
    """Workgroups enough for whole rounds over the chip, the widest tiles ending behind N."""
    counts = np.random.default_rng(4).poisson(6, 256).tolist()
    for K, N in ((64, 640), (320, 640), (1088, 320)):
        print(K, N, flush=True)
        _run(*_case(counts, 64, K, N, "none", x4, True, seed=K))


@pytest.mark.parametrize("counts,N", [([9, 2], 64), ([90, 40], 64), ([90, 40, 70, 80], WIDE)])
@pytest.mark.parametrize("x4", [False, True])
def test_product_extreme_scales(counts, N, x4):
    """Scale bytes 0 and 254, and 255 (NaN) in one column of one weight and one row of x."""
    K = 192
    dev, ref, tol = _case(counts, 20, K, N, "none", x4, False, seed=2)
    dev["w"].scales[0, 5] = 0
    dev["w"].scales[1, 6, 2] = 255
    dev["w"].codes[1, 6, 32:48] = 0           # a block of zeros under a NaN scale is NaN too
    if x4:
        dev["x"].scales[1] = 255
    out = mx.product(**dev).double().cpu().numpy()
    nan = np.zeros_like(ref, bool)
    nan[counts[0]:counts[0] + counts[1], 6] = True
    if x4:
        nan[1] = True
    assert np.array_equal(np.isnan(out), nan)
    keep = ~nan
    keep[:counts[0], 5] = False
    assert (np.abs(out - ref)[keep] <= tol[keep]).all()
    tiny = np.abs(out[:counts[0], 5])[~nan[:counts[0], 5]]
    assert (tiny < 2.0 ** -100).all()
    # 2^127 against 2^-127: products of ordinary size
    if x4:
        dev["x"].scales.fill_(0)
        dev["w"].scales.fill_(254)
    else:
        dev["x"].mul_(2.0 ** -100)
        dev["w"].scales.fill_(227)
    out = mx.product(**dev).double().cpu().numpy()
    xv = (R.mx_values(dev["x"].codes.cpu().numpy(), dev["x"].scales.cpu().numpy()) if x4
          else dev["x"].double().cpu().numpy())
    lo = 0
    for e, c in enumerate(counts):
        v = R.mx_values(dev["w"].codes[e].cpu().numpy(), dev["w"].scales[e].cpu().numpy()).T
        want, m = xv[lo:lo + c] @ v, np.abs(xv[lo:lo + c]) @ np.abs(v)
        assert (np.abs(out[lo:lo + c] - want) <= np.abs(want) * 2.0 ** -8 * 1.01 + (K + 16) * R.U32 * m).all()
        lo += c


def test_product_row_of_x_with_nan_stays_alone():
    """A NaN or infinite row of x reaches its own slots only, also where its tile pads rows."""
    for counts, N in (([6, 0, 3], 64), ([100, 45], 64), ([100, 45, 70, 80], WIDE)):
        dev, ref, tol = _case(counts, 10, 128, N, "none", False, False, seed=4)
        dev["x"][2, 7] = float("nan")
        dev["x"][counts[0], 1] = float("inf")
        out = mx.product(**dev).double().cpu().numpy()
        hit = np.zeros(len(ref), bool)
        hit[[2, counts[0]]] = True
        assert (~np.isfinite(out[2])).all() and (~np.isfinite(out[counts[0]])).any()
        assert (np.abs(out - ref)[~hit] <= tol[~hit]).all()


@pytest.mark.parametrize("N", [192, WIDE])
def test_product_same_bits_again_in_a_graph_and_on_another_stream(N):
    dev, ref, tol = _case([30, 0, 200, 7], 60, 256, N, "swiglu", False, True, seed=6)
    want = mx.product(**dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mx.product(**dev, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mx.product(**dev)
    for i in range(3):
        dev["x"].mul_(0.5)
        want = mx.product(**dev)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


# ---- the layer on 4-bit experts ---------------------------------------------------------------

def _layer(T, d, f, E, act, seed=0):
    g = torch.Generator().manual_seed(seed)

    def rnd(*s, std):
        return (torch.randn(*s, generator=g) * std).to(BF).cuda()

    return (rnd(T, d, std=1.0), rnd(E, d, std=0.05), rnd(E, d, f, std=d ** -0.5),
            rnd(E, d, f, std=d ** -0.5) if act == "swiglu" else None, rnd(E, f, d, std=f ** -0.5))


@pytest.mark.parametrize("T,d,f,E,k", [(1, 256, 320, 8, 2), (40, 192, 448, 16, 4), (700, 256, 384, 8, 2)])
@pytest.mark.parametrize("act", ["swiglu", "silu", "relu"])
@pytest.mark.parametrize("rows", ["bf16", "mx"])
def test_layer_on_quantised_experts(T, d, f, E, k, act, rows):
    """mx.forward against the same steps in 64 bits on the quantised values: h and the
    combined y are rounded to bfloat16 on the way (2e-2 of the largest, the layer's own
    tolerance); with 4-bit rows from the very codes that the calls make."""
    x, wg, w1, w3, w2 = _layer(T, d, f, E, act)
    q = mx.quantize_experts(w1, w3, w2)
    y = mx.forward(x, wg, None, q, k, True, act, rows).double().cpu().numpy()
    ids, gates, _ = layer._route(x, wg, None, E, k, True, 0)
    counts, offsets, eti, tim, _ = layer._maps(ids, T, E, k)
    xr = mx.quantize(x) if rows == "mx" else x
    h = mx.product(xr, q.w1, offsets, eti, q.w3 if act == "swiglu" else None, act)
    hr = mx.quantize(h) if rows == "mx" else h
    hv = (R.mx_values(*(t.cpu().numpy() for t in hr)) if rows == "mx" else hr.double().cpu().numpy())
    off, tm, gt = offsets.cpu().numpy(), tim.cpu().numpy(), gates.double().cpu().numpy()
    O = np.zeros((T * k, d))
    for e in range(E):
        O[off[e]:off[e + 1]] = hv[off[e]:off[e + 1]] @ R.mx_values(q.w2.codes[e].cpu().numpy(), q.w2.scales[e].cpu().numpy()).T
    want = (gt[:, :, None] * O[tm]).sum(1)
    assert np.abs(y - want).max() <= 2e-2 * np.abs(want).max()
    if rows == "bf16":
        # and the whole layer on the dequantised weights
        deq = [None if t is None else mx.dequantize(t).transpose(1, 2).contiguous() for t in q]
        y2, _ = layer.forward(x, wg, None, *deq, k, True, act=act)
        y2 = y2.double().cpu().numpy()
        assert np.abs(y - y2).max() <= 2e-2 * np.abs(y2).max()


def test_layer_on_quantised_experts_in_a_graph():
    x, wg, w1, w3, w2 = _layer(48, 256, 320, 16, "swiglu")
    q = mx.quantize_experts(w1, w3, w2)
    mx.forward(x, wg, None, q, 4, True, rows="mx")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mx.forward(x, wg, None, q, 4, True, rows="mx")
    for i in range(3):
        x.mul_(0.9)
        want = mx.forward(x, wg, None, q, 4, True, rows="mx")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    assert mx.forward(x[:0], wg, None, q, 4, True).shape == (0, 256)
