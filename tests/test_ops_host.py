"""The operators that take no model, without a GPU: what their entry points refuse, the 4-bit quantiser, and the plain forms that the
GPU tests compare with."""
import ctypes

import numpy as np
import pytest

import paper_2007_11794_amd as rn
from ops_reference import distill_row, q4_weights, sample_row

EINVAL, ERANGE, EWORKSPACE = -1, -4, -5
BUF = ctypes.create_string_buffer(1 << 16)
AT = (ctypes.addressof(BUF) + 255) // 256 * 256


def at(offset):
    return ctypes.c_void_p(AT + offset)


def q4(B=2, V=4, H=40, group=32, codes=at(0), code_ld=20, st=0, scale=at(1024), zero=None, bias=None, xt=0, x=at(2048), x_ld=40, yt=0, y=at(4096), y_ld=4):
    return rn.lib().rnnlm_q4_matvec(B, V, H, group, codes, code_ld, st, scale, zero, bias, xt, x, x_ld, yt, y, y_ld, None)


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), EINVAL), (dict(V=0), EINVAL), (dict(H=0), EINVAL), (dict(group=16), EINVAL), (dict(group=256), EINVAL), (dict(group=0), EINVAL),
    (dict(st=2), EINVAL), (dict(xt=-1), EINVAL), (dict(yt=7), EINVAL), (dict(H=65537, code_ld=40000, x_ld=70000), ERANGE),
    (dict(V=(1 << 30) + 1, y_ld=1 << 31), ERANGE), (dict(code_ld=19), EINVAL), (dict(x_ld=39), EINVAL), (dict(y_ld=3), EINVAL), (dict(codes=None), EINVAL),
    (dict(scale=None), EINVAL), (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(scale=at(1025)), EINVAL), (dict(x=at(2050)), EINVAL), (dict(y=at(4098)), EINVAL),
    (dict(bias=at(3)), EINVAL), (dict(y=at(0)), EINVAL), (dict(y=at(2048)), EINVAL), (dict(y=at(1024)), EINVAL), (dict(zero=at(4100)), EINVAL),
    (dict(bias=at(4096)), EINVAL), (dict(code_ld=1 << 41), EINVAL), (dict(B=0, codes=None, scale=None, x=None, y=None), 0)])
def test_q4_refusals(change, status):
    assert q4(**change) == status


def sample(N=2, V=8, dtype=0, z=at(0), ld=8, T=None, k=None, p=None, m=None, u=at(1024), word=at(2048), lp=at(3328), ws=at(4096), wsb=1 << 15):
    return rn.lib().rnnlm_sample(N, V, dtype, z, ld, T, k, p, m, u, word, lp, ws, wsb, None)


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), EINVAL), (dict(V=0), EINVAL), (dict(dtype=2), EINVAL), (dict(ld=7), EINVAL), (dict(z=None), EINVAL), (dict(u=None), EINVAL), (dict(word=None), EINVAL),
    (dict(ws=None), EWORKSPACE), (dict(wsb=8), EWORKSPACE), (dict(ws=at(4100)), EWORKSPACE), (dict(z=at(2)), EINVAL), (dict(u=at(1)), EINVAL), (dict(T=at(1026)), EINVAL),
    (dict(word=at(0)), EINVAL), (dict(word=at(1024)), EINVAL), (dict(lp=at(2052)), EINVAL), (dict(ws=at(0)), EINVAL), (dict(T=at(2048)), EINVAL), (dict(k=at(3328)), EINVAL),
    (dict(V=(1 << 30) + 1, ld=1 << 31), ERANGE), (dict(N=(1 << 24) + 1), ERANGE), (dict(N=0, z=None, u=None, word=None, ws=None), 0)])
def test_sample_refusals(change, status):
    assert sample(**change) == status


def distill(N=2, V=8, K=3, dtype=0, z=at(0), ld=8, tw=at(1024), tl=at(1280), label=None, T=1.0, a=0.0, g=None, loss=at(2048), stats=at(2304), grad=None, gld=0, ws=at(4096),
            wsb=1 << 15):
    return rn.lib().rnnlm_distill(N, V, K, dtype, z, ld, tw, tl, label, T, a, g, loss, stats, grad, gld, ws, wsb, None)


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), EINVAL), (dict(V=0), EINVAL), (dict(K=-1), EINVAL), (dict(dtype=3), EINVAL), (dict(ld=7), EINVAL), (dict(z=None), EINVAL), (dict(tw=None), EINVAL),
    (dict(tl=None), EINVAL), (dict(T=0.0), EINVAL), (dict(T=-1.0), EINVAL), (dict(T=float("nan")), EINVAL), (dict(T=float("inf")), EINVAL), (dict(a=0.5), EINVAL),
    (dict(a=-0.1, label=at(1536)), EINVAL), (dict(a=1.5, label=at(1536)), EINVAL), (dict(a=float("nan"), label=at(1536)), EINVAL), (dict(loss=None), EINVAL),
    (dict(stats=None), EINVAL), (dict(grad=at(512), gld=7), EINVAL), (dict(ws=None), EWORKSPACE), (dict(wsb=8), EWORKSPACE), (dict(ws=at(4104)), EWORKSPACE),
    (dict(loss=at(0)), EINVAL), (dict(stats=at(2048)), EINVAL), (dict(grad=at(32), gld=8), EINVAL), (dict(grad=at(0), gld=9), EINVAL), (dict(grad=at(1024), gld=8), EINVAL),
    (dict(grad=at(0), gld=8, loss=at(60)), EINVAL), (dict(z=at(2)), EINVAL), (dict(V=(1 << 30) + 1, ld=1 << 31), ERANGE), (dict(N=0, z=None, loss=None, stats=None, ws=None), 0)])
def test_distill_refusals(change, status):
    assert distill(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(grad=None), EINVAL), (dict(stats=None), EINVAL), (dict(grad=at(32)), EINVAL), (dict(stats=at(512)), EINVAL), (dict(T=0.0), EINVAL), (dict(N=0, grad=None), 0),
    (dict(gld=7), EINVAL), (dict(grad=at(2)), EINVAL)])
def test_distill_backward_refusals(change, status):
    a = dict(N=2, z=at(0), stats=at(2304), grad=at(512), gld=8, T=1.0)
    a.update(change)
    assert rn.lib().rnnlm_distill_backward(a["N"], 8, 3, 0, a["z"], 8, at(1024), at(1280), None, a["T"], 0.0, None, a["stats"], a["grad"], a["gld"], None) == status


def test_workspaces():
    for f in (rn.rnnlm_sample_workspace_bytes, rn.rnnlm_distill_workspace_bytes):
        assert f(0, 10) == 0 and f(10, 0) == 0 and f(-1, 10) == 0 and f(10, -1) == 0
        assert 0 < f(1, 1) <= f(1024, 200000)


def test_binding_refuses_what_is_not_a_device_tensor():
    import torch
    f, i = torch.zeros, torch.int32
    with pytest.raises(TypeError):
        rn.rnnlm_q4_matvec(f(4, 16, dtype=torch.uint8), f(1, 4), 32, f(2, 32), f(2, 4), stream=0)
    with pytest.raises(TypeError):
        rn.rnnlm_sample(f(2, 8), f(2), f(2, dtype=i), f(2), f(4096, dtype=torch.uint8), stream=0)
    with pytest.raises(TypeError):
        rn.rnnlm_distill(f(2, 8), f(2, 3, dtype=i), f(2, 3), f(2), f(2, 4), f(4096, dtype=torch.uint8), stream=0)


@pytest.mark.parametrize("V,H,group", [(1, 1, 32), (7, 33, 32), (5, 100, 64), (3, 256, 128), (4, 129, 128)])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantiser(V, H, group, zeros):
    rng = np.random.default_rng(V * 1000 + H)
    w = rng.standard_normal((V, H)).astype(np.float32)
    w[0, : min(H, group)] = 0.0                                              # a group of zeros
    if V > 3:
        w[3] = np.abs(w[3])
    codes, scales, zero = rn.rnnlm_q4_quantize(w, group, zeros)
    back = q4_weights(codes, H, group, scales, zero)
    of = np.arange(H) // group
    # nearest code: half a step; the zero point is rounded too, which moves the ends of the range by half a step more and its codes by none
    assert (np.abs(back - w) <= scales.T[:, of] * ((1.0 if zeros else 0.5) + 1e-6)).all()
    assert (back[0, : min(H, group)] == 0).all()
    if H % 2:
        assert (codes[:, -1] >> 4 == 0).all()
    if not zeros:
        groups = [w[:, g * group:(g + 1) * group] for g in range(scales.shape[0])]
        assert all((np.abs(x).max(1) / np.float32(7) == pytest.approx(s, rel=1e-6)) for x, s in zip(groups, scales))


def test_quantiser_refusals():
    w = np.ones((2, 40), np.float32)
    with pytest.raises(TypeError):
        rn.rnnlm_q4_quantize(w, 48)
    for bad in (np.nan, np.inf, -np.inf):
        w[1, 39] = bad
        with pytest.raises(rn.RnnlmError):
            rn.rnnlm_q4_quantize(w, 32)


def test_plain_draw_on_a_row_done_by_hand():
    z = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    assert [sample_row(z, u)[0] for u in (0.0, 0.05, 0.15, 0.55, 0.75, 0.95)] == [0, 0, 1, 2, 3, 4]
    assert [sample_row(z, u, k=3)[0] for u in (0.0, 0.49, 0.51, 0.76)] == [1, 1, 2, 3]       # 0.4, 0.2, 0.2
    assert [sample_row(z, u, k=2)[0] for u in (0.0, 0.66, 0.67)] == [1, 1, 2]                # of equal ones the lower id
    assert [sample_row(z, u, p=0.55)[0] for u in (0.6, 0.7)] == [1, 2]
    assert sample_row(z, 0.99, p=0.3)[0] == 1 and sample_row(z, 0.99, m=0.9)[0] == 1 and sample_row(z, 0.99, T=0.0)[0] == 1
    assert sample_row(z, 0.99, p=-1.0)[0] == 1 and sample_row(z, 0.99, m=7.0)[0] == 1
    assert sample_row([-np.inf, -np.inf], 0.5)[0] == -1 and sample_row([1.0, np.nan], 0.5)[0] == -1


@pytest.mark.parametrize("T,a", [(1.0, 0.0), (2.0, 0.3), (0.7, 1.0)])
def test_plain_gradient_against_differences(T, a):
    rng = np.random.default_rng(5)
    V, K, e = 23, 6, 1e-5
    z, words, t = rng.standard_normal(V) * 2, np.array([3, 7, -1, 3, 20, 11]), rng.standard_normal(K)
    _, grad, _ = distill_row(z, words, t, 4, T, a)
    for i in range(V):
        up, down = z.copy(), z.copy()
        up[i] += e
        down[i] -= e
        # the second difference's error is e^2 / 6 times a third derivative below T^-1 + 1 in magnitude; rounding is 2^-52 * 10 / e
        assert abs((distill_row(up, words, t, 4, T, a)[0] - distill_row(down, words, t, 4, T, a)[0]) / (2 * e) - grad[i]) < 1e-9


def test_more_teacher_entries_than_a_list_holds():
    assert distill(K=4097) == ERANGE and distill(N=0, K=4096) == 0


def test_interleaved_rows_are_no_overlap():
    """Rows of the gradient in the gaps of the logits' rows: nothing is shared, and nothing but the workspace is refused."""
    assert distill(z=at(0), ld=16, grad=at(32), gld=16, ws=None) == EWORKSPACE
    assert distill(z=at(0), ld=16, grad=at(28), gld=16, ws=at(4096)) == EINVAL
    assert distill(z=at(0), ld=16, grad=at(68), gld=16, ws=at(4096)) == EINVAL
    assert distill(z=at(0), ld=16, grad=at(32), gld=17, ws=at(4096)) == EINVAL


@pytest.mark.parametrize("change,status", [(dict(tw=at(1025)), EINVAL), (dict(tl=at(1282)), EINVAL), (dict(label=at(1537), a=0.5), EINVAL), (dict(g=at(1795)), EINVAL),
                                           (dict(N=(1 << 21) + 1), ERANGE)])
def test_distill_refuses_misaligned_lists_and_too_many_rows(change, status):
    assert distill(**change) == status


def test_sample_refuses_more_rows_than_a_grid_holds():
    assert sample(N=(1 << 21) + 1) == ERANGE
