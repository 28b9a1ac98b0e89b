"""The byte count that `bench.py --layer` reports for its norms is the floor that perf/operators.py states for the same call."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "perf"))

import bench  # noqa: E402
import operators  # noqa: E402


@pytest.mark.parametrize("B,N,C,kept", [(32, 321, 512, 119), (8, 8192, 512, 1413), (1, 3, 64, 3)])
def test_bytes_of_the_norms(B, N, C, kept):
    case = operators._norm("", "layer", B, N, C, "bf16", "rms", "rms", B, ",".join([str(kept)] * B))
    parameters = 2 * 4 * C * (B + 3)
    assert bench.layer_norm_bytes(B * kept, B, N, C) == operators.work(case)["bytes"] - parameters
