"""Head rotation, appends, reads and attention over the 4-bit cache at their edges: orders of access within a block, values that are
not finite beside turned elements, values beyond a half, empty pools, rows laid over others.

Oracles and tolerances are those of test_packed_cache.py and test_serving.py, where they are derived; what differs is said at the test.
"""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import packed_ref as pref
from paper_2506_04708_b200 import binding, build as lib_build, inputs
from tests import test_packed_cache as tp
from tests import test_serving as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_04708_b200", "csrc")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


# ---------------------------------------------------------------- order within a block
def _body(source, head):
    """The text between the braces that follow `head`, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, source)).read())
    at = text.index("{", text.index(head))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at + 1:i]
    raise AssertionError(head)


def test_what_a_block_shares_of_its_range_is_written_before_its_last_barrier():
    """Other warps read these members without a barrier of their own, so no write to them may follow the last one here."""
    body = _body("attention_split.cuh", "ta_begin(const TaSplit& p")
    last = body.rindex("__syncthreads()")
    written = {m.group(1): m.start() for m in re.finditer(r"\bsh\.(\w+)(?:\[[^\]]*\])?\s*=[^=]", body)}
    assert set(written) == {"sum", "b", "b_start", "total", "groups"}
    assert all(at < last for at in written.values()), written
