"""Distillation at the borders of its forms, workspaces and numbers, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2007_11794_amd as rn
from ops_reference import distill_row
from test_gpu_distill import backward, case, check, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_workspace_of_many_rows_serves_the_last_few():
    """As in training: made for the largest batch, used for a shorter one at the end."""
    V = 70001
    ws = torch.empty(rn.rnnlm_distill_workspace_bytes(60, V), dtype=torch.uint8, device=DEV)
    for N in (60, 48, 47, 5, 1):
        d = case(N, V, 9)
        loss, stats, grad = torch.empty(N, device=DEV), torch.empty((N, 4), device=DEV), torch.empty((N, V), device=DEV)
        rn.rnnlm_distill(d["z"], d["words"], d["t"], loss, stats, ws, temperature=2.0, labels=d["label"], label_weight=0.25, row_weight=d["g"], grad=grad)
        torch.cuda.synchronize()
        check(d, 2.0, 0.25, loss, grad, rows=range(0, N, 12))


@pytest.mark.parametrize("T", [1e-45, 1e-40, 4e-39, 1e-38, 1e-30, 1e-20, 1e-10, 1e10, 1e18])
@pytest.mark.parametrize("N,V", [(6, 3000), (2, 70001), (60, 70001)])
def test_temperatures_of_any_size(N, V, T):
    """A loss of T times something of order one: where that is below the normal numbers, its two last roundings are half a least step, 2^-150, each."""
    t = float(np.float32(T))
    for a in (0.0, 0.25):
        d = case(N, V, 40)
        loss, stats, grad = run(d, T, a)
        only = run(d, T, a, grad=False)[0]
        wanted = torch.full((N,), np.nan, dtype=torch.float64)
        for n in range(0, N, 10):
            want, _, far = distill_row(d["z"][n].double().cpu().numpy(), d["words"][n].cpu().numpy(), d["t"][n].double().cpu().numpy(), int(d["label"][n]), t, a)
            r = 2.0 ** -18 + (V / 256 + 16) * 2.0 ** -24
            bar = (t * t * (1 - a) + a) * (r + 2.0 ** -20 * far) + 2.0 ** -22 * abs(want) + 2 * 2.0 ** -150
            assert abs(float(loss[n]) - want) <= bar and abs(float(only[n]) - want) <= bar, (n, float(loss[n]), float(only[n]), want)
            wanted[n] = want
        check(d, T, a, wanted, grad, rows=range(0, N, 10))
        check(d, T, a, wanted, backward(d, T, a, stats), rows=range(0, N, 10))


@pytest.mark.parametrize("T", [0.5, 1.0, 2e37, 1e38, 3e38])
@pytest.mark.parametrize("N,V,dtype", [(6, 3000, torch.float32), (6, 3000, torch.bfloat16), (2, 70001, torch.float32), (60, 70001, torch.float32), (20, 140000, torch.bfloat16)])
def test_logits_further_apart_than_the_largest_number(N, V, dtype, T):
    """Shares at such temperatures are of order one; a loss beyond the largest float is infinite."""
    t = float(np.float32(T))
    rng = np.random.default_rng(V)
    d = case(N, V, 40, dtype)
    d["z"] = torch.from_numpy((rng.uniform(-1, 1, (N, V)) * 3.3e38).astype(np.float32)).to(DEV).to(dtype)
    d["t"] = torch.from_numpy((rng.uniform(-1, 1, (N, 40)) * 3.3e38).astype(np.float32)).to(DEV)
    rows = range(0, N, 10)
    for a in (0.0, 0.25, 1.0):
        loss, stats, grad = run(d, T, a)
        only = run(d, T, a, grad=False)[0]
        wanted = torch.full((N,), np.nan, dtype=torch.float64)
        for n in rows:
            want, _, far = distill_row(d["z"][n].double().cpu().numpy(), d["words"][n].cpu().numpy(), d["t"][n].double().cpu().numpy(), int(d["label"][n]), t, a)
            bar = (t * t * (1 - a) + a) * (2.0 ** -18 + (V / 256 + 16) * 2.0 ** -24 + 2.0 ** -20 * far) + 2.0 ** -22 * abs(want)
            for got in (float(loss[n]), float(only[n])):
                assert got == np.inf if want - bar > 3.4028235e38 else abs(got - want) <= bar or (got == np.inf and want + bar > 3.4028235e38), (n, a, got, want)
            wanted[n] = want
        check(d, T, a, wanted, grad, rows=rows)
        check(d, T, a, wanted, backward(d, T, a, stats), rows=rows)
