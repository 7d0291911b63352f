"""Calls at the edges of what the operators around the layer take."""
import numpy as np
import pytest
import torch

from paper_2601_05296_amd import mx
from tests.test_gpu_mx import WIDE, _case

pytestmark = pytest.mark.gpu


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
