"""The gated delta rule's step refuses a result that shares memory with another array, without a GPU: its wavefronts would
read what others have written.  The result may lie in the place of v itself, and between other arrays of one buffer."""
import pytest

from paper_1805_11144_amd import mergesim as MS
from test_memory_operators_cpu import step
from test_operators_cpu import refused

ROWS, HK, H, DK, DV, SLOTS = 2, 2, 4, 24, 40, 4   # the sizes of step()
FAR = {n: (i + 1) << 24 for i, n in enumerate(("q", "k", "v", "decay", "rate", "state", "slots", "y"))}
ORDER = ("q", "k", "v", "decay", "rate", "state", "slots", "y")


def call(kw, **at):
    return step(**kw), *[dict(FAR, **at)[n] for n in ORDER]


def passes(kw, **at):
    """Goes on to the device, which is not there: an error of the runtime, not a refusal, and nothing is launched."""
    code = MS.load_library().ms_gated_delta_step(*call(dict(kw, device=10000), **at))
    assert code != 0 and "overlap" not in MS.load_library().ms_last_error().decode()


E = 4   # float32
Y_END, Q_END, MATRIX = ROWS * H * DV * E, ROWS * HK * DK * E, H * DK * DV * E


@pytest.mark.parametrize("kw,at", [
    ({}, dict(y=FAR["q"])), ({}, dict(y=FAR["k"])), ({}, dict(y=FAR["decay"])), ({}, dict(y=FAR["rate"])),
    ({}, dict(y=FAR["slots"])), ({}, dict(y=FAR["state"])), ({}, dict(y=FAR["state"] + SLOTS * MATRIX - E)),
    ({}, dict(y=FAR["q"] + Q_END - E)), ({}, dict(y=FAR["q"] - Y_END + E)), ({}, dict(y=FAR["v"] + E)),
    ({}, dict(y=FAR["v"] + DV * E)), (dict(v_stride=(2 * H * DV, DV)), dict(y=FAR["v"])),
    (dict(v_stride=(H * DV, 2 * DV)), dict(y=FAR["v"])),
    # columns of one buffer of 500 values a row, one too near
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"] + (H * DV - 1) * E)),
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"] + (500 - H * DV + 1) * E)),
    (dict(q_stride=(500, DK), y_stride=(500, DV)), dict(y=FAR["q"] + (HK * DK - 1) * E)),
    (dict(decay_stride=(500, 1), y_stride=(500, DV)), dict(y=FAR["decay"] + 3 * E)),
    # head by head beside each other, one too near
    (dict(v_stride=(800, 100), y_stride=(800, 100)), dict(y=FAR["v"] + 39 * E)),
    (dict(v_stride=(800, 100), y_stride=(800, 100)), dict(y=FAR["v"] + 61 * E))])
def test_refused(kw, at):
    refused("ms_gated_delta_step", *call(kw, **at), words="overlap")


@pytest.mark.parametrize("kw,at", [
    ({}, {}), ({}, dict(y=FAR["v"])), ({}, dict(y=FAR["q"] + Q_END)), ({}, dict(y=FAR["q"] - Y_END)),
    ({}, dict(y=FAR["state"] + SLOTS * MATRIX)), (dict(n_slots=0), dict(y=FAR["state"])), ({}, dict(slots=None)),
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"])),
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"] + H * DV * E)),
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"] + (500 - H * DV) * E)),
    (dict(v_stride=(500, DV), y_stride=(500, DV)), dict(y=FAR["v"] - H * DV * E)),
    (dict(q_stride=(500, DK), y_stride=(500, DV)), dict(y=FAR["q"] + HK * DK * E)),
    (dict(decay_stride=(500, 1), y_stride=(500, DV)), dict(y=FAR["decay"] + 4 * E)),
    (dict(v_stride=(800, 100), y_stride=(800, 100)), dict(y=FAR["v"] + 40 * E)),
    (dict(v_stride=(800, 100), y_stride=(800, 100)), dict(y=FAR["v"] + 60 * E)),
    (dict(v_stride=(100, 800), y_stride=(100, 800)), dict(y=FAR["v"] + 40 * E)),
    (dict(rows=1, v_stride=(7, DV)), dict(y=FAR["v"]))])
def test_passed_on(kw, at):
    passes(kw, **at)
