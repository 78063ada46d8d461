"""The operators around the decoding step at the ends of their arguments: bounds, devices, values that are not finite, small
weights, layouts, aliases, streams.  Tolerances as in test_serving.py unless a test derives its own.
"""
import os
import subprocess

import numpy as np
import pytest

from paper_2506_04708_b200 import binding, build as lib_build, inputs
from tests import test_serving as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------- the visibility mask
@pytest.fixture(scope="module")
def bounds_program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("bounds") / "attention_bounds")
    subprocess.run([lib_build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe,
                    os.path.join(ROOT, "tests", "attention_bounds.cu")], check=True)
    return exe


@pytest.mark.parametrize("N,group", [(1, 1), (64, 7), (200, 2), (513, 1), (33, 5), (640, 1), (640, 5), (18, 7), (19, 7), (3, 128), (2, 130), (65, 3)])
@pytest.mark.parametrize("own", [0, 1])
def test_the_mask_is_read_for_existing_nodes_only(bounds_program, N, group, own):
    """Both kernels ask attn_nodes_seen for each row of their row tiles, rows beyond the last node among them.  The mask ends
    where the mapping does; the words are those of the definition."""
    for masked in (1, 0):
        run = subprocess.run([bounds_program, str(N), str(group), "3", str(own), str(masked)], capture_output=True, text=True, timeout=60)
        assert run.returncode == 0, (run.returncode, run.stdout)
