"""Distillation against the definition in 64 bits: loss, statistics and gradient, at once and apart, masks, short lists, labels, odd rows."""
import numpy as np
import pytest
import torch

import paper_2007_11794_amd as rn
from ops_reference import distill_row

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


def case(N, V, K, dtype=torch.float32, label=True, seed=0, spread=3.0):
    rng = np.random.default_rng(seed + 31 * V + K)
    d = {"z": torch.from_numpy((rng.standard_normal((N, V)) * spread).astype(np.float32)).to(DEV).to(dtype)}
    words = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(N)]).astype(np.int32).reshape(N, K)
    d["words"] = torch.from_numpy(words).to(DEV)
    d["t"] = torch.from_numpy((rng.standard_normal((N, K)) * 3).astype(np.float32)).to(DEV)
    d["label"] = torch.from_numpy(rng.integers(-1, V, N).astype(np.int32)).to(DEV) if label else None
    d["g"] = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).to(DEV)
    return d


def run(d, T, a, grad=True, weight=True, out=None):
    N, V = d["z"].shape
    loss, stats = torch.full((N,), 7.0, device=DEV), torch.full((N, 4), 7.0, device=DEV)
    ws = torch.randint(0, 256, (rn.rnnlm_distill_workspace_bytes(N, V),), dtype=torch.uint8, device=DEV)
    if out is None and grad:
        out = torch.full((N, V), 7.0, device=DEV, dtype=d["z"].dtype)
    rn.rnnlm_distill(d["z"], d["words"], d["t"], loss, stats, ws, temperature=T, labels=d["label"], label_weight=a, row_weight=d["g"] if weight else None, grad=out)
    torch.cuda.synchronize()
    return loss, stats, out


def backward(d, T, a, stats, out=None):
    out = torch.full(d["z"].shape, 7.0, device=DEV, dtype=d["z"].dtype) if out is None else out
    rn.rnnlm_distill_backward(d["z"], d["words"], d["t"], stats, out, temperature=T, labels=d["label"], label_weight=a, row_weight=d["g"])
    torch.cuda.synchronize()
    return out


def check(d, T, a, loss, grad, weight=True, rows=None):
    """A sum of exponentials is good to r = 2^-18 (2^-24 of an exponent's argument, up to 40 where it counts, the instruction's own last
    place) and 2^-24 for each of the V / 256 additions of a thread; logarithms and shares follow it."""
    z = d["z"].double().cpu().numpy()
    V = z.shape[1]
    T = float(np.float32(T))
    a = float(np.float32(a))
    r = 2.0 ** -18 + (V / 256 + 16) * 2.0 ** -24
    words, t = d["words"].cpu().numpy(), d["t"].double().cpu().numpy()
    label = np.full(len(z), -1) if d["label"] is None else d["label"].cpu().numpy()
    g = d["g"].double().cpu().numpy() if weight else np.ones(len(z))
    loss = loss.double().cpu().numpy()
    half = 0.0 if grad is None else torch.finfo(grad.dtype).eps / 2
    grad = None if grad is None else grad.double().cpu().numpy()
    for n in rows if rows is not None else range(len(z)):
        want, dz, far = distill_row(z[n], words[n], t[n], label[n], T, a)
        if not np.isfinite(want):
            assert np.isnan(loss[n]) if np.isnan(want) else loss[n] == want, (n, loss[n], want)
        else:
            assert abs(loss[n] - want) <= (T * T * (1 - a) + a) * (r + 2.0 ** -20 * far) + 2.0 ** -22 * abs(want), (n, loss[n], want)
        if grad is None:
            continue
        dz = dz * g[n]
        if np.isnan(dz).any():
            assert np.isnan(grad[n]).all(), n
            continue
        # p and the teacher's share of each word to r and 2^-23 of the argument
        size = np.abs(g[n]) * (1 - a) * T * share(z[n], T, r)
        for w, q in zip(*teacher(words[n], t[n], T)):
            size[w] += np.abs(g[n]) * (1 - a) * T * q * r
        if label[n] >= 0:
            size += np.abs(g[n]) * a * share(z[n], 1.0, r)
            size[label[n]] += np.abs(g[n]) * a * 2.0 ** -22
        bar = half * np.abs(dz) + (1 + half) * (size + 2.0 ** -22 * np.abs(dz)) + 2.0 ** -126
        off = np.abs(grad[n] - dz)
        assert (off <= bar).all(), (n, int(np.argmax(off / bar)), (off / bar).max())


def share(z, T, r):
    with np.errstate(invalid="ignore"):
        y = (z - z.max()) / T
        p = np.exp(y)
        return np.where(p > 0, p / p.sum() * (r + 2.0 ** -22 * np.where(np.isfinite(y), np.abs(y), 0.0)), 0.0)


def teacher(words, t, T):
    on = words >= 0
    if not on.any() or not t[on].max() > -np.inf:
        return [], []
    q = np.exp((t[on] - t[on].max()) / T)
    return words[on], q / q.sum()


SIZES = [(1, 1, 1), (1, 2, 2), (3, 7, 5), (2, 64, 64), (5, 255, 16), (4, 256, 1), (8, 1000, 16), (3, 1027, 300), (40, 4099, 33), (2, 8192, 64), (3, 8193, 64), (300, 3001, 20), (7, 20011, 1000),
         (2, 65536, 100), (5, 65537, 3), (2, 131075, 50), (3, 200003, 257)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_sizes(N, V, K, dtype):
    for T, a, label in ((1.0, 0.0, False), (2.0, 0.3, True)):
        d = case(N, V, K, dtype, label)
        loss, stats, grad = run(d, T, a)
        check(d, T, a, loss, grad)
        only, stats2, _ = run(d, T, a, grad=False)
        check(d, T, a, only, None)
        check(d, T, a, loss, backward(d, T, a, stats))
        check(d, T, a, loss, backward(d, T, a, stats2))
        z = d["z"].double()
        top = z.amax(1, keepdim=True)
        want = torch.cat([top, 1 / torch.exp((z - top) / T).sum(1, keepdim=True), 1 / torch.exp(z - top).sum(1, keepdim=True), torch.zeros_like(top)], 1)
        for s in (stats, stats2):
            assert bool(((s.double() - want).abs() <= (2.0 ** -18 + (V / 256 + 16) * 2.0 ** -24) * want.abs()).all())


@pytest.mark.parametrize("T", [0.1, 1.0, 5.0, 40.0])
@pytest.mark.parametrize("a", [0.0, 0.5, 1.0])
def test_temperatures_and_weights(T, a):
    d = case(6, 3000, 40)
    loss, stats, grad = run(d, T, a)
    check(d, T, a, loss, grad)
    check(d, T, a, loss, backward(d, T, a, stats))
    loss, _, grad = run(d, T, a, weight=False)
    check(d, T, a, loss, grad, weight=False)


def masked(dtype):
    """Rows with something missing or wrong in each."""
    V, K = 2500, 12
    d = case(24, V, K, dtype)
    z, w, t, y = d["z"], d["words"], d["t"], d["label"]
    y[:] = torch.arange(24, device=DEV, dtype=torch.int32) * 7
    low = torch.finfo(dtype).min
    free = [i for i in range(V) if i not in set(w.flatten().tolist()) | set(y.tolist())]
    z[0, free[:500]] = -INF
    z[1, free] = low
    z[2, int(w[2, 3])] = -INF                                     # a teacher's word that the student cannot say
    z[3, int(y[3])] = -INF
    z[4] = -INF
    z[5, 9] = NAN
    z[6, 11] = INF
    w[7] = -1
    t[8] = -INF
    t[9, 2:] = -INF
    w[10, ::2] = -1
    t[10, ::2] = NAN                                               # not looked at
    w[11] = -1
    y[11] = -1                                                     # nothing to learn
    w[12] = -1
    y[12] = -1
    z[12, 3] = NAN                                                 # nor looked at
    y[13] = -1
    w[14, 5] = V
    w[15, 5] = -2
    y[16] = V
    y[17] = -2
    t[18, 4] = NAN
    t[19, 4] = INF
    w[20] = w[20, 0].clone()                                       # one word, many times
    w[21, 6:] = w[21, :6].clone()
    t[22] = torch.finfo(torch.float32).min
    z[23] = low
    return d


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,a", [(1.0, 0.5), (3.0, 0.0), (2.0, 1.0)])
def test_what_is_missing_or_wrong(dtype, T, a):
    d = masked(dtype)
    loss, stats, grad = run(d, T, a)
    check(d, T, a, loss, grad)
    check(d, T, a, loss, backward(d, T, a, stats))
    loss, stats, _ = run(d, T, a, grad=False)
    check(d, T, a, loss, backward(d, T, a, stats))


def test_a_repeated_word_gives_one_gradient_every_time():
    d = case(4, 900, 64)
    d["words"][:] = d["words"][:, :1]
    grads = [run(d, 2.0, 0.2)[2] for _ in range(5)]
    assert all(torch.equal(grads[0], g) for g in grads)


def test_no_teacher_entries_at_all():
    d = case(5, 700, 0)
    loss, stats, grad = run(d, 2.0, 0.4)
    check(d, 2.0, 0.4, loss, grad)
    check(d, 2.0, 0.4, loss, backward(d, 2.0, 0.4, stats))


def test_gradient_against_differences_of_the_loss():
    V, T, a, e = 37, 2.0, 0.3, 1e-4
    d = case(2, V, 9)
    _, _, grad = run(d, T, a, weight=False)
    z, words, t, label = d["z"].double().cpu().numpy(), d["words"].cpu().numpy(), d["t"].double().cpu().numpy(), d["label"].cpu().numpy()
    a = float(np.float32(a))
    for n in range(2):
        for i in range(V):
            up, down = z[n].copy(), z[n].copy()
            up[i] += e
            down[i] -= e
            slope = (distill_row(up, words[n], t[n], label[n], T, a)[0] - distill_row(down, words[n], t[n], label[n], T, a)[0]) / (2 * e)
            assert abs(float(grad[n, i]) - slope) <= 1e-6          # e^2 / 6 times third derivatives of order 1; 2^-18 of shares below 0.2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_strides_and_nothing_beside(dtype):
    N, K = 7, 20
    for V in (9, 1001, 70001):
        d = case(N, V, K, dtype) if V > K else case(N, V, 5, dtype)
        want = run(d, 2.0, 0.25)
        wide = torch.full((N, V + 6), 7.0, device=DEV, dtype=dtype)
        for off in (0, 1, 3):
            z = wide[:, off:off + V]
            z.copy_(d["z"])
            e = dict(d, z=z)
            out = torch.full((N + 2, V + 9), 7.0, device=DEV, dtype=dtype)
            got = run(e, 2.0, 0.25, out=out[1:N + 1, 5 - off:5 - off + V])
            check(e, 2.0, 0.25, got[0], got[2])
            got[2].fill_(7.0)
            assert bool((out == 7).all())
            got = run(e, 2.0, 0.25, out=z)                         # over the logits themselves
            check(d, 2.0, 0.25, got[0], got[2])
            z.copy_(d["z"])
            check(d, 2.0, 0.25, want[0], backward(e, 2.0, 0.25, want[1], out=z))
            z.fill_(7.0)
            assert bool((wide == 7).all())


def test_rows_beyond_two_gigabytes():
    V, ld = 1500, 1 << 30
    d = case(3, V, 10)
    z = torch.as_strided(torch.empty(2 * ld + V, device=DEV), (3, V), (ld, 1))
    z.copy_(d["z"])
    d["z"] = z
    out = torch.as_strided(torch.empty(2 * ld + V, device=DEV), (3, V), (ld, 1))
    loss, stats, grad = run(d, 2.0, 0.5, out=out)
    check(d, 2.0, 0.5, loss, grad)
    out.fill_(0)
    check(d, 2.0, 0.5, loss, backward(d, 2.0, 0.5, stats, out=out))


@pytest.mark.parametrize("N,V", [(3, 60000), (400, 1000)])
def test_another_stream_and_a_graph(N, V):
    ds = [case(N, V, 12, seed=s) for s in range(3)]
    want = [run(d, 2.0, 0.3) for d in ds]
    b = {k: v.clone() for k, v in ds[0].items()}
    loss, stats, grad, back = torch.empty(N, device=DEV), torch.empty((N, 4), device=DEV), torch.empty((N, V), device=DEV), torch.empty((N, V), device=DEV)
    ws = torch.empty(rn.rnnlm_distill_workspace_bytes(N, V), dtype=torch.uint8, device=DEV)

    def both():
        rn.rnnlm_distill(b["z"], b["words"], b["t"], loss, stats, ws, temperature=2.0, labels=b["label"], label_weight=0.3, row_weight=b["g"], grad=grad)
        rn.rnnlm_distill_backward(b["z"], b["words"], b["t"], stats, back, temperature=2.0, labels=b["label"], label_weight=0.3, row_weight=b["g"])

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert torch.equal(loss, want[0][0]) and torch.equal(grad, want[0][2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in (1, 2, 0, 1):
        for k in b:
            b[k].copy_(ds[i][k])
        loss.zero_()
        grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[i][0]) and torch.equal(grad, want[i][2])
        check(ds[i], 2.0, 0.3, loss, back, rows=range(0, N, max(1, N // 8)))
        again = run(ds[2], 2.0, 0.3)
        assert torch.equal(again[0], want[2][0]) and torch.equal(again[2], want[2][2])


def test_no_rows():
    e, i = torch.empty, torch.int32
    rn.rnnlm_distill(e((0, 9), device=DEV), e((0, 3), dtype=i, device=DEV), e((0, 3), device=DEV), e(0, device=DEV), e((0, 4), device=DEV), None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("N,V,K", [(3, 5000, 4096), (2, 70001, 4096), (130, 9000, 2000), (2, 100000, 1500)])
def test_long_lists(N, V, K):
    d = case(N, V, K)
    d["words"][0, 100:200] = d["words"][0, :100].clone()           # and words that repeat in one of them
    loss, stats, grad = run(d, 2.0, 0.25)
    check(d, 2.0, 0.25, loss, grad, rows=range(min(N, 4)))
    check(d, 2.0, 0.25, loss, backward(d, 2.0, 0.25, stats), rows=range(min(N, 4)))


def test_a_row_that_weighs_nothing():
    d = case(3, 3000, 20)
    d["g"][1] = 0.0
    loss, stats, grad = run(d, 2.0, 0.3)
    check(d, 2.0, 0.3, loss, grad)
    assert bool((grad[1] == 0).all()) and bool((backward(d, 2.0, 0.3, stats)[1] == 0).all())
