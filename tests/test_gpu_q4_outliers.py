"""Products with 4-bit weights where one unit of a row is millions of times as large as the others."""
import numpy as np
import pytest
import torch

from ops_reference import q4_weights
from test_gpu_q4 import call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", [1e4, 1e6, 1e8])
@pytest.mark.parametrize("B,V,H,group,zero", [(1, 400, 512, 32, False), (3, 400, 512, 32, True), (16, 400, 500, 64, False), (5, 400, 512, 64, True), (1, 400, 512, 128, False),
                                              (9, 400, 300, 128, True), (40, 20000, 200, 64, False), (40, 20000, 200, 32, True), (64, 66000, 96, 128, True), (64, 66000, 96, 64, False),
                                              (64, 66000, 96, 32, False)])
def test_a_unit_far_above_the_others(B, V, H, group, zero, large):
    """Every second word does not see that unit (its code is the zero point): what the others give it is good to their own bits, as in 32 bits.  Bars as in
    test_gpu_q4.check, but for the small units: 2^-23 of themselves or 2^-50 of the row's largest."""
    d = make(B, V, H, group, zero=zero, bias=False)
    at = 37
    zeros = np.full((-(-H // group), V), 8, np.uint8) if d["zeros"] is None else d["zeros"].cpu().numpy()
    codes = d["codes"].cpu().numpy()
    codes[::2, at // 2] = (codes[::2, at // 2] & 0x0F) | (zeros[at // group, ::2] << 4)
    d["codes"] = torch.from_numpy(codes).to(d["codes"].device)
    d["x"][:, at] *= large
    rows = [0, B // 2, B - 1]
    out = call(d)[rows].double().cpu().numpy()
    w = q4_weights(codes, H, group, d["scales"].double().cpu().numpy(), zeros)
    assert (w[::2, at] == 0).all()
    x = d["x"].double().cpu().numpy()[rows]
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    half = 2.0 ** -24
    bar = half * np.abs(want) + (1 + half) * ((2 ** -22 + (H + 16) * 2 ** -24) * size + 2 ** -50 * np.abs(x).max(1, keepdims=True) * np.abs(w).sum(1))
    off = np.abs(out - want)
    assert (off <= bar).all(), (off / bar).max()
