"""Products with 4-bit weights against 64-bit sums: types, group sizes, zero points, odd sizes, strides, alignments, infinities."""
import numpy as np
import pytest
import torch

import paper_2007_11794_amd as rn
from ops_reference import q4_weights, unpack_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(B, V, H, group, x="f32", scale="f32", zero=False, bias=True, pad=0, shift=0, seed=0):
    """pad: bytes more than a row of codes needs; shift: bytes the codes start behind an aligned address."""
    rng = np.random.default_rng(seed + 7919 * V + H)
    row, groups = (H + 1) // 2, -(-H // group)
    d = {"H": H, "group": group}
    flat = torch.from_numpy(rng.integers(0, 256, V * (row + pad) + shift, dtype=np.uint8)).to(DEV)
    d["codes"] = flat[shift:].view(V, row + pad)[:, :row]
    d["scales"] = torch.from_numpy(rng.uniform(0.005, 0.015, (groups, V)).astype(np.float32)).to(DEV).to(TYPES[scale])
    d["zeros"] = torch.from_numpy(rng.integers(0, 256 if zero == "wide" else 16, (groups, V), dtype=np.uint8)).to(DEV) if zero else None
    d["bias"] = torch.from_numpy(rng.standard_normal(V).astype(np.float32)).to(DEV) if bias else None
    d["x"] = torch.from_numpy(rng.standard_normal((B, H)).astype(np.float32)).to(DEV).to(TYPES[x])
    return d


def call(d, y="f32", out=None, x=None):
    x = d["x"] if x is None else x
    if out is None:
        out = torch.full((x.shape[0], d["codes"].shape[0]), float("nan"), device=DEV, dtype=TYPES[y])
    rn.rnnlm_q4_matvec(d["codes"], d["scales"], d["group"], x, out, zeros=d["zeros"], bias=d["bias"])
    torch.cuda.synchronize()
    return out


def check(d, out, rows=None):
    """Half a step of y's type, 2^-23 of every product for the two terms of x (2^-38 of the row's largest at least) and for its
    product with a scale, and 2^-24 of the magnitudes for each of H + 16 additions."""
    H = d["H"]
    w = q4_weights(d["codes"].cpu().numpy(), H, d["group"], d["scales"].double().cpu().numpy(), None if d["zeros"] is None else d["zeros"].cpu().numpy())
    x = d["x"].double().cpu().numpy()
    bias = 0.0 if d["bias"] is None else d["bias"].double().cpu().numpy()
    if rows is not None:
        x, out = x[rows], out[rows]
    want, size = x @ w.T + bias, np.abs(x) @ np.abs(w).T + np.abs(bias)
    half = torch.finfo(out.dtype).eps / 2
    bar = half * np.abs(want) + (1 + half) * ((2 ** -22 + (H + 16) * 2 ** -24) * size + 2 ** -38 * np.abs(x).max(1, keepdims=True) * np.abs(w).sum(1))
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bar).all(), (off - bar).max()


SIZES = [(1, 1, 1, 32), (1, 5, 31, 32), (2, 16, 32, 32), (3, 17, 33, 64), (1, 1000, 64, 32), (4, 1003, 100, 32), (15, 333, 127, 128), (16, 64, 128, 128),
         (17, 515, 129, 64), (31, 130, 250, 32), (33, 1029, 256, 128), (64, 257, 320, 64), (65, 77, 96, 32), (130, 200, 512, 128), (5, 40, 1500, 64), (3, 20, 8200, 128), (40, 33, 5000, 32)]


@pytest.mark.parametrize("B,V,H,group", SIZES)
@pytest.mark.parametrize("x,y,scale,zero", [("f32", "f32", "f32", False), ("bf16", "bf16", "bf16", True), ("f32", "bf16", "bf16", "wide"), ("bf16", "f32", "f32", True)])
def test_sizes_and_types(B, V, H, group, x, y, scale, zero):
    d = make(B, V, H, group, x=x, scale=scale, zero=zero, bias=V % 2 == 1)
    check(d, call(d, y))


@pytest.mark.parametrize("B,V,H,group", [(1, 20011, 512, 128), (16, 20011, 512, 64), (61, 9001, 256, 32), (8, 100003, 100, 32), (300, 3001, 192, 64)])
def test_many_words(B, V, H, group):
    d = make(B, V, H, group, zero=True)
    check(d, call(d))


@pytest.mark.parametrize("B,V,H", [(17, 33001, 96), (33, 22003, 33), (47, 30010, 130), (100, 10007, 260), (33, 131085, 64), (70, 65553, 129), (200, 32771, 100)])
@pytest.mark.parametrize("x,y,group,zero", [("f32", "f32", 32, True), ("f32", "f32", 64, False), ("f32", "f32", 128, True), ("bf16", "bf16", 32, False), ("bf16", "f32", 64, True),
                                            ("bf16", "bf16", 128, False)])
def test_many_rows_of_many_words(B, V, H, x, y, group, zero):
    """Sizes at which a workgroup takes 32 or 64 rows.  Rows at the blocks' edges are compared."""
    d = make(B, V, H, group, x=x, zero=zero, pad=V % 3)
    check(d, call(d, y), rows=[b for b in (0, 15, 16, 31, 32, 63, 64, 99, 127, 128, 199, B - 1) if b < B])


def test_rows_of_larger_blocks_do_not_depend_on_each_other():
    for x in ("f32", "bf16"):
        d = make(70, 65601, 64, 32, x=x)
        whole = call(d)
        for b in (0, 31, 32, 64, 69):
            assert torch.equal(call(d, x=d["x"][b:b + 1])[0], whole[b])


@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 0), (0, 1), (3, 2), (14, 0), (14, 6), (30, 16), (62, 9)])
@pytest.mark.parametrize("H", [34, 100, 260])
def test_rows_of_codes_anywhere(pad, shift, H):
    for V in (1, 3, 50):
        d = make(3, V, H, 32, pad=pad, shift=shift)
        check(d, call(d))


def test_strides_of_rows_and_nothing_beside_them():
    B, V, H = 5, 77, 90
    d = make(B, V, H, 32)
    wide = torch.full((B, H + 9), float("nan"), device=DEV)
    wide[:, 4:4 + H] = d["x"]
    d["x"] = wide[:, 4:4 + H]
    for y in ("f32", "bf16"):
        out = torch.full((B + 2, V + 5), 7.0, device=DEV, dtype=TYPES[y])
        call(d, out=out[1:B + 1, 3:3 + V])
        check(d, out[1:B + 1, 3:3 + V])
        out[1:B + 1, 3:3 + V] = 7.0
        assert bool((out == 7).all())


def test_rows_do_not_depend_on_each_other():
    d = make(70, 301, 200, 64)
    whole = call(d)
    for b in (0, 15, 16, 33, 64, 69):
        alone = call(d, x=d["x"][b:b + 1])
        assert torch.equal(alone[0], whole[b])


def test_magnitudes():
    """Rows of very large and very small numbers, and rows that hold both: what is small is good to 2^-39 of the largest."""
    d = make(6, 65, 96, 32, bias=False)
    d["x"][0] *= 1e30
    d["x"][1] *= 1e-30
    d["x"][2, ::2] *= 1e8
    d["x"][3] = 0.0
    d["x"][4, 5:] = 0.0
    d["x"][5, ::3] *= 1e-6
    out = call(d)
    check(d, out)
    assert bool((out[3] == 0).all())
    b = make(2, 65, 96, 32, x="bf16", bias=False)
    b["x"][0] *= 1e30
    b["x"][1, ::2] *= 1e6
    check(b, call(b))


def test_largest_numbers():
    d = make(2, 33, 64, 32, bias=False)
    d["x"][0] = 0.0
    d["x"][0, 3] = 3.4e38
    d["x"][1] = 2.0 ** -140                                       # below the smallest normal number
    out = call(d).double().cpu().numpy()
    w = q4_weights(d["codes"].cpu().numpy(), 64, 32, d["scales"].double().cpu().numpy(), None)
    want = d["x"].double().cpu().numpy() @ w.T
    assert (np.abs(out[0] - want[0]) <= 2 ** -20 * np.abs(want[0])).all()
    assert (np.abs(out[1] - want[1]) <= 2 ** -20 * np.abs(want[1]) + 2 ** -140).all()


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_row(x):
    d = make(20, 100, 130, 32, x=x)
    clean = d["x"].clone()
    for row, value in ((1, float("inf")), (4, float("-inf")), (17, float("nan"))):
        d["x"][row, 77] = value
    out = call(d)
    q = unpack_codes(d["codes"].cpu().numpy(), 130)[:, 77] - 8
    with np.errstate(invalid="ignore"):
        for row, value in ((1, np.inf), (4, -np.inf)):
            assert np.array_equal(out[row].cpu().numpy(), (value * q).astype(np.float32), equal_nan=True)
    assert bool(out[17].isnan().all())
    d["x"] = clean
    check(d, out, rows=[i for i in range(20) if i not in (1, 4, 17)])


def test_codes_behind_an_odd_row_do_not_count():
    d = make(2, 9, 35, 32)
    a = call(d)
    d["codes"][:, -1] ^= 0xF0
    assert torch.equal(call(d), a)


def test_codes_beyond_two_gigabytes():
    V, H = 70, 64
    big = torch.zeros(V * (1 << 25), dtype=torch.uint8, device=DEV)         # 2.3 GB: the last rows start beyond 31 bits
    d = make(3, V, H, 32)
    codes = big.view(V, 1 << 25)[:, :H // 2]
    codes.copy_(d["codes"])
    d["codes"] = codes
    check(d, call(d))


def test_another_stream_and_a_graph():
    d = make(5, 3001, 200, 64)
    x = [torch.randn((5, 200), device=DEV) for _ in range(3)]
    want = [call(d, x=v) for v in x]
    side = torch.cuda.Stream()
    out, buf = torch.empty((5, 3001), device=DEV), x[0].clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        rn.rnnlm_q4_matvec(d["codes"], d["scales"], 64, buf, out, bias=d["bias"])
    side.synchronize()
    assert torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rn.rnnlm_q4_matvec(d["codes"], d["scales"], 64, buf, out, bias=d["bias"])
    for i in (1, 2, 0, 1):
        buf.copy_(x[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        assert torch.equal(call(d, x=x[2]), want[2])


def test_no_rows():
    d = make(1, 10, 32, 32)
    rn.rnnlm_q4_matvec(d["codes"], d["scales"], 32, torch.empty((0, 32), device=DEV), torch.empty((0, 10), device=DEV))
    torch.cuda.synchronize()


def test_quantised_model_gives_the_logits_of_its_rounded_weights():
    rng = np.random.default_rng(3)
    w = (rng.standard_normal((500, 100)) * 0.1).astype(np.float32)
    for zeros in (False, True):
        codes, scales, zero = rn.rnnlm_q4_quantize(w, 64, zeros)
        d = {"H": 100, "group": 64, "codes": torch.from_numpy(codes).to(DEV), "scales": torch.from_numpy(scales).to(DEV), "bias": None,
             "zeros": torch.from_numpy(zero).to(DEV) if zeros else None, "x": torch.from_numpy(rng.random((4, 100)).astype(np.float32)).to(DEV)}
        check(d, call(d))
