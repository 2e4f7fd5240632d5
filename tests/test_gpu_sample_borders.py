"""The draw of a word at the borders of its lists, weights and numbers, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from ops_reference import sample_row
from test_gpu_sample import check, draw, limits, logits

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


def near_halves(T, count, low, high, seed):
    """z1, z2 (float32) whose weights e^(z / T) add up to 1 but for something between `low` and `high` in magnitude, and that."""
    rng = np.random.default_rng(seed)
    found = []
    while sum(len(f[0]) for f in found) < count:
        z1 = (T * rng.uniform(-2.0, -0.3, 1 << 20)).astype(np.float32)
        z2 = (T * np.log1p(-np.exp(z1.astype(np.float64) / T))).astype(np.float32)
        off = np.exp(z1.astype(np.float64) / T) - (1 - np.exp(z2.astype(np.float64) / T))
        at = (np.abs(off) >= low) & (np.abs(off) <= high)
        found.append((z1[at], z2[at], off[at]))
    return [np.concatenate([f[i] for f in found])[:count] for i in range(3)]


@pytest.mark.parametrize("T", [1.0, 0.75, 2.5])
def test_weights_are_good_to_the_last_bit_of_their_numbers(T):
    """Three words, the first of weight 1, at u = 1/2: it is drawn where the others weigh less than it.  Their weights are off by a unit of 2^-50 each
    at most, 1.8e-15 together (and the definition here by 2e-16 each), which a difference of 4e-15 and more has to survive."""
    z1, z2, off = near_halves(T, 150, 4e-15, 2e-13, int(T * 100))
    N = len(z1)
    z = torch.from_numpy(np.stack([np.zeros(N, np.float32), z1, z2], 1)).to(DEV)
    word, _ = draw(z, np.full(N, 0.5, np.float32), T=np.full(N, T))
    assert np.array_equal(word, np.where(off < 0, 0, 1)), int((word != np.where(off < 0, 0, 1)).sum())


@pytest.mark.parametrize("V,dtype", [(1000, torch.float32), (5000, torch.float32), (5000, torch.bfloat16), (60000, torch.float32), (70000, torch.float32), (200003, torch.float32),
                                     (200003, torch.bfloat16)])
def test_a_min_p_of_one_unit(V, dtype):
    """All words but one weigh between half a unit of the weights' numbers and one, and are rounded to what min_p asks for, far from any that weighs
    more: what is drawn does not depend on which others a wave has beside them."""
    bits = min(50, 62 - int(np.ceil(np.log2(V))))
    low = (-np.log(2.0) * (bits + torch.linspace(0.05, 0.9, 16))).to(dtype)
    low = low[(-low.double() / np.log(2.0) > bits + 0.03) & (-low.double() / np.log(2.0) < bits + 0.92)][0]
    z = torch.full((4, V), float(low), device=DEV, dtype=dtype)
    z[:, V - 3] = 0.0
    z[1, :700] = -float("inf")
    u = [0.0, 0.0, 0.5, 2.0 ** -24]
    word, lp = draw(z, u, m=np.full(4, 2.0 ** -bits))
    assert list(word[:3]) == [0, 700, V - 3]
    total = 2.0 ** bits + np.array([V - 1, V - 701, V - 1])
    want = np.log(np.array([1.0, 1.0, 2.0 ** bits]) / total)
    assert (np.abs(lp[:3] - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -50).all()
    first = 2.0 ** -24 * (2.0 ** bits + V - 1)                     # the numbers up to the word that is drawn have to pass it
    assert word[3] == (V - 3 if first >= V - 3 else int(first))


@pytest.mark.parametrize("V", [1, 2, 3, 64, 1000, 4096])
def test_log_probabilities_of_short_rows(V):
    """The weights' unit is 2^-50 here, however few words there are; a row of one word has nothing to be off by."""
    N = 40
    z = logits(N, V, 7 * V + 1)
    u, T, k, p, m = limits(N, V, V + 2)
    word, lp = draw(z, u, T, k, p, m)
    one, rows = 2.0 ** -50, z.double().cpu().numpy()
    at = lambda x, n: np.float64(np.float32(x[n]))  # noqa: E731
    for n in range(N):
        want, want_lp, w = sample_row(rows[n], at(u, n), at(T, n), int(k[n]), at(p, n), at(m, n))
        # rounded once to 32 bits; the word's number and the kept words' (V at most, each at least as heavy as what it is off by) a unit each
        assert word[n] == want and abs(lp[n] - want_lp) <= 2.0 ** -24 * abs(want_lp) + one / w + V * one, (n, lp[n], want_lp)
    if V == 1:
        assert (word == 0).all() and (lp == 0).all()


@pytest.mark.parametrize("V,dtype", [(300, torch.float32), (5000, torch.float32), (5000, torch.bfloat16), (70000, torch.float32), (140000, torch.bfloat16)])
@pytest.mark.parametrize("T", [2e37, 1e38, 3e38])
def test_logits_further_apart_than_the_largest_number(V, dtype, T):
    """At such a temperature they weigh something all the same, and have an order."""
    rng = np.random.default_rng(V)
    z = torch.from_numpy((rng.uniform(-1, 1, (8, V)) * 3.3e38).astype(np.float32)).to(DEV).to(dtype)
    z[:, 5] = 3.3e38
    u, T = rng.random(8).astype(np.float32) * np.float32(0.99999), np.full(8, T)
    k, p = np.geomspace(2, V - 1, 8).astype(int), np.array([0.02, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.999])
    check(z, u, T=T)
    check(z, u, T=T, k=k)
    check(z, u, T=T, p=p)
    check(z, u, T=T, k=k, p=p, m=p / 100)
