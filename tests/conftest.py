import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

# Tests that hold a value which is not the right one, kept as they are, and why.
WRONG = {
    "tests/test_gpu_policy.py::test_loss_scales_beyond_the_logits_type":
        "expects the gradient cut to float16 before the loss scale multiplies it; of its 3,600 entries 47 % are then more "
        "than half a unit of float16 off the 64-bit gradient times the scale.  "
        "test_a_loss_scale_lifts_what_the_logits_type_could_not_hold holds the gradient to that.",
}


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (HIP device) and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running CPU test")


def pytest_collection_modifyitems(items):
    for item in items:
        if item.nodeid in WRONG:
            item.add_marker(pytest.mark.xfail(reason=WRONG[item.nodeid], raises=AssertionError, strict=False))
