"""Sizes that the operators without a model work out on the host and in their kernels: the library's own header, compiled for the host, and
the queries of the built library."""
import ctypes

import pytest

import paper_2007_11794_amd as rn
from test_host_plan import check_on_the_host
from test_ops_host import EINVAL, EWORKSPACE, at, distill, q4, sample


def test_sizes_of_the_operators_on_the_host(tmp_path):
    check_on_the_host(tmp_path, "operators_check")


def test_a_workspace_serves_fewer_rows_and_words_too():
    rows = list(range(1, 70)) + [100, 256, 1000, 1024, 4096, 1 << 21]
    words = [1, 1000, 49151, 49152, 65536, 65537, 70000, 131072, 131073, 200000, 262144, 300000, 1000000, 1 << 24, 1 << 30]
    for f in (rn.rnnlm_sample_workspace_bytes, rn.rnnlm_distill_workspace_bytes):
        for V in words:
            needs = [f(N, V) for N in rows]
            assert needs == sorted(needs), V
        for N in rows:
            needs = [f(N, V) for V in words]
            assert needs == sorted(needs), N


def test_a_call_asks_for_no_more_than_it_uses():
    """One row of 65536 words is cut into segments, 49 rows are not: those pass the check of the workspace with 16 bytes of it (and are refused
    here for a loss within the logits)."""
    assert distill(N=1, V=65536, ld=65536, loss=at(0), wsb=16) == EWORKSPACE
    assert distill(N=49, V=65536, ld=65536, loss=at(0), wsb=16) == EINVAL


FAR = ctypes.c_void_p(1 << 46)                                     # (nothing is read: the calls below are refused)


@pytest.mark.parametrize("call", [lambda ld: q4(B=1 << 24, x=FAR, x_ld=ld), lambda ld: q4(B=2, V=1 << 29, codes=FAR, code_ld=ld, y=FAR, y_ld=1 << 29),
                                  lambda ld: q4(B=1 << 24, y=FAR, y_ld=ld), lambda ld: sample(N=1 << 21, z=FAR, ld=ld), lambda ld: distill(N=1 << 21, z=FAR, ld=ld),
                                  lambda ld: distill(N=1 << 21, z=FAR, ld=1 << 20, grad=FAR, gld=ld)])
def test_rows_whose_bytes_pass_63_bits_are_refused(call):
    assert call(1 << 40) == EINVAL
