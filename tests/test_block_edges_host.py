"""CPU checks at the edges of what the operators around the layer take."""
import torch

from paper_2601_05296_amd import binding as B
from paper_2601_05296_amd import grads, layer

FAKE = 1 << 20   # aligned, never dereferenced


def test_norm_bwd_of_no_rows_needs_no_gate_gradient():
    """The gradient of a token's or a full gate has no element then; an empty tensor's address
    is NULL. A channel's is summed over the rows, and written."""
    lib = B.load_library()

    def bwd(flags, dgate):
        return lib.moe_norm_bwd(None, None, None, None, None, None, None, None, None, 1.0, 0, 64, flags, None,
                                None, dgate, None, None, None, 0, None)

    tok, chan = B.MOE_GATE_TOKEN, B.MOE_GATE_CHANNEL
    for fl in (tok, tok | chan, tok | B.MOE_F32):
        assert bwd(fl, None) == B.MOE_OK and bwd(fl, FAKE) == B.MOE_OK
    assert bwd(chan, None) == B.MOE_ERR_INVALID_ARG and b"dgate is NULL" in lib.moe_last_error()
    assert bwd(0, FAKE) == B.MOE_ERR_INVALID_ARG and b"dgate without" in lib.moe_last_error()


def test_gradients_of_parameters_alone():
    """What layer.backward(keep=True) adds beside the parameters' gradients stays out of a norm."""
    par = {n: torch.ones(3) for n in ("dw1", "dw3", "dw2", "dw_gate")}
    rest = {n: torch.ones(5) for n in ("dx", "dX_slot", "dx_ffn", "d_gates")}
    assert [t.numel() for t in grads._list({**rest, **par})] == [3] * 4
    assert [t.numel() for t in grads._list([{**par, **rest}, rest, par["dw1"]])] == [3] * 5


def test_no_tokens_make_no_chunk():
    for want in (1, 4, 100):
        assert list(layer._chunks(0, layer.aligned_chunk(want, 0))) == []


def test_quantize_refuses_what_no_launch_covers():
    """Sizes whose grid would need 2^32 threads: refused before the launch, not failed by it."""
    lib = B.load_library()

    def quant(batch, rows, K, flags=0):
        return lib.moe_mx_quantize(FAKE, batch, rows, K, flags, FAKE, FAKE, None)

    assert quant(1, (1 << 31) - 1, 32) == B.MOE_ERR_UNSUPPORTED and b"2^36 - 4096" in lib.moe_last_error()
    assert quant(1, (1 << 31) - 127, 32, B.MOE_F32) == B.MOE_ERR_UNSUPPORTED
    for rows in ((1 << 29) - 126, (1 << 29) - 2):
        assert quant(1, rows, 32, B.MOE_TRANSPOSED) == B.MOE_ERR_UNSUPPORTED and b"2^29 - 128" in lib.moe_last_error()


def test_product_refuses_results_over_its_inputs():
    lib = B.load_library()
    far = 1 << 30

    def gemm(x=far, xs=None, w=2 * far, ws=3 * far, w3=4 * far, ws3=5 * far, off=6 * far, rows=7 * far, out=FAKE):
        return lib.moe_mx_gemm(x, xs, w, ws, w3, ws3, off, rows, 4, 8, 64, 128, 2, B.MOE_GATED, out, None)

    # out 2048 bytes; x 512 (256 and 8 in 4 bits), weights 8192 and 512 each, offsets 12, rows 32
    for name, size in (("x", 512), ("w", 8192), ("ws", 512), ("w3", 8192), ("ws3", 512), ("off", 12), ("rows", 32)):
        what = {"ws": "w_scales", "ws3": "w3_scales", "off": "offsets"}.get(name, name)
        for at in (FAKE, FAKE + 2032, FAKE - (size - 1) // 16 * 16):
            assert gemm(**{name: at}) == B.MOE_ERR_INVALID_ARG, (name, at)
            assert b"out overlaps " + what.encode() in lib.moe_last_error()
    assert gemm(xs=FAKE + 16) == B.MOE_ERR_INVALID_ARG and b"x_scales" in lib.moe_last_error()
