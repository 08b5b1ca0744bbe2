import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that hold a value which their operator's definition does not give; they stay as they were written, and are expected to fail.
WRONG_VALUES = {
    "test_head_where_every_class_is_masked_by_the_lowest_value":
        "asserts a loss of 0 where the softmax of equal logits has log(classes); "
        "tests/test_gpu_training_edges.py::test_the_softmax_of_equal_logits_however_low holds that",
}


def pytest_collection_modifyitems(config, items):
    for item in items:
        if item.name in WRONG_VALUES:
            item.add_marker(pytest.mark.xfail(reason=WRONG_VALUES[item.name], strict=True))
    # GPU tests are skipped (not failed) where no device is visible, so that a
    # plain `pytest tests/` works on a CPU-only machine.
    try:
        import torch
        have_gpu = torch.cuda.is_available()
    except Exception:
        have_gpu = False
    if have_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU visible")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
