"""Sizes that the operators without a model work out on the host and in their kernels: the library's own header, compiled for the host."""
from test_host_plan import check_on_the_host


def test_sizes_of_the_operators_on_the_host(tmp_path):
    check_on_the_host(tmp_path, "operators_check")
