import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU")


# Tests that expect a value that is wrong, and why.
WRONG = {
    "test_gpu_attention_grad.py::test_keys_that_are_not_there":
        "drops entries of the list outside [0, n) from the gradient, where thin_attention clamps "
        "them to the nearest row (test_keys_without_weight_hold_anything has the clamped form)",
}


def pytest_collection_modifyitems(config, items):
    for item in items:
        reason = WRONG.get(f"{item.path.name}::{getattr(item, 'originalname', item.name)}")
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, raises=AssertionError, strict=True))
    # GPU tests are skipped (not failed) where there is no GPU, so that
    # `pytest tests/` works anywhere; the round-end runs select `-m gpu` explicitly.
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU visible")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
