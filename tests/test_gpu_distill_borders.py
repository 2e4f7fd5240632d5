"""Distillation at the borders of its forms, workspaces and numbers, against the definition in 64 bits."""
import pytest
import torch

import paper_2007_11794_amd as rn
from test_gpu_distill import case, check

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
