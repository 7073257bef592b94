"""Scales and rates of the operators that a double holds and a float32 does not are refused, without a GPU: they
would reach the kernels as infinities."""
import ctypes as C

import pytest

from paper_1805_11144_amd import mergesim as MS
from test_operators_cpu import A, embed, orth, refused


@pytest.mark.parametrize("scale", [1e300, -1e300, 3.5e38])
def test_scales(scale):
    refused("ms_embed", embed(scale=scale), A, A, A, words="scale")
    refused("ms_embed_grad", embed(scale=scale), A, A, A, A, 1 << 30, words="scale")
    refused("ms_embed_grad_workspace", embed(scale=scale), C.byref(C.c_int64()), words="scale")


@pytest.mark.parametrize("rule", [(1e300, 0.9, 0.0), (0.1, 1e300, 0.0), (1e30, 0.9, 1e30), (0.1, 0.9, 1e300)])
def test_rates(rule):
    refused("ms_orthogonal_update", orth(), MS.OrthRule(*rule, 1), A, A, A, A, 1 << 40, words="finite")


def test_the_largest_float_is_not_refused():
    assert MS.load_library().ms_embed_grad_workspace(embed(scale=3.4e38), C.byref(C.c_int64())) == 0
