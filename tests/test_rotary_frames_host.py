"""Rotary plans by frame, row and column: what numbers of tokens they take.  A plan without frames
has a position for each axis of a row, one with frames a single one, and the binding counts them by the
plan: numbers that the library takes for "no frames" are refused before there is a plan.  No GPU."""
import os
import shutil

import pytest


@pytest.fixture(scope="module")
def ec():
    if not shutil.which("nvcc") and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2608_02474_gb300 import build
    build.build()
    from paper_2608_02474_gb300 import echocache
    return echocache


@pytest.mark.parametrize("frame", [(0, 0), (0, 6), (-24, 6), (24, 0), (24, -6), (24, 7), (2 ** 31, 6), (24,), (24, 6, 1)])
def test_bad_frames(ec, frame):
    with pytest.raises(ValueError, match="frame"):
        ec.Rotary(64, [12, 10, 10], frame=frame, device="cpu")


@pytest.mark.parametrize("pairs", [[32], [16, 16], [8, 8, 8, 8], 32])
def test_frames_have_three_axes(ec, pairs):
    with pytest.raises(ValueError, match="frame"):
        ec.Rotary(64, pairs, frame=(24, 6), device="cpu")


def test_positions_of_a_row(ec):
    for pairs, frame, columns in (([12, 10, 10], (24, 6), 1), ([12, 10, 10], None, 3), (32, None, 1), ([8, 8], None, 2),
                                  ([12, 0, 10], (6, 6), 1)):
        plan = ec.Rotary(64, pairs, frame=frame, device="cpu")
        assert plan.columns == columns and plan.cstruct.frame_tokens == (frame[0] if frame else 0)
