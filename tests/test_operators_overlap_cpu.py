"""The gated lowpass refuses strides by which rows of its result overlap, without a GPU: two rows would write the
same place."""
import pytest

from paper_1805_11144_amd import mergesim as MS
from test_operators_cpu import A, gated, refused


@pytest.mark.parametrize("kw", [
    dict(y_stride=(8, 8)), dict(y_stride=(16, 8)), dict(y_stride=(8, 15)), dict(y_stride=(70000 * 8 - 1, 8)),
    dict(y_stride=(7, 16), steps=1), dict(batch=3, y_stride=(8, 16)), dict(batch=3, y_stride=(16, 39)),
    dict(steps=2, y_stride=((1 << 40) - 1, 7)), dict(steps=(1 << 31) - 1, y_stride=(1 << 39, 1 << 39))])
def test_overlapping_rows(kw):
    refused("ms_gated_lowpass", gated(**kw), A, A, A, A, A, A, A, A, 1 << 50, words="overlap")


@pytest.mark.parametrize("kw", [
    dict(y_stride=(70000 * 8, 8)), dict(y_stride=(8, 16)), dict(batch=3, y_stride=(16, 40)), dict(batch=1, y_stride=(0, 8)),
    dict(steps=1, y_stride=(8, 0)), dict(steps=0, y_stride=(0, 1))])
def test_others_reach_the_next_check(kw):
    """A misaligned pointer, which is looked at later."""
    refused("ms_gated_lowpass", gated(**kw), A, A, A + 2, A, A, A, A, A, 1 << 50, words="aligned")


def test_strides_of_a_gradient_may_repeat():
    """dy is only read: one row for all steps is what a sum over steps hands back."""
    refused("ms_gated_lowpass_grad", gated(y_stride=(8, 0)), A, A, A, A, A, A, A + 2, A, A, A, 1 << 50, words="aligned")
