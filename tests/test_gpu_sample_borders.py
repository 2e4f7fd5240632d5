"""The draw of a word at the borders of its lists, weights and numbers, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("V,dtype", [(65537, torch.float32), (100000, torch.float32), (190000, torch.float32), (140000, torch.bfloat16), (180000, torch.bfloat16)])
@pytest.mark.parametrize("tied", [8192, 8193, 10000, 12288, 12289])
def test_more_words_of_one_logit_than_a_list_holds(V, dtype, tied):
    """Around the length of a row's list and what of it goes to LDS; the words that are counted and not listed are drawn all the same."""
    rng = np.random.default_rng(V + tied)
    z = torch.from_numpy((rng.standard_normal((3, V)) - 8).clip(None, -1).astype(np.float32)).to(DEV).to(dtype)
    for n in range(3):
        z[n, torch.from_numpy(rng.choice(V, tied, replace=False)).to(DEV)] = 3.0
    u = np.array([0.03, 0.6, 0.97], np.float32)
    check(z, u, k=[50, 3000, tied - 1])
    check(z, u, p=[0.9, 0.2, 0.6])
    check(z, u, k=[40, 4000, 2000], p=[0.5, 0.9, 0.7])
    check(z[:1], u[1:2], p=[0.5])
