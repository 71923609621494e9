import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


# Cases whose expected value is wrong.  Mode tail, lists of the whole vocabulary that add up to Q = 1 + 5e-5: the loss is
# sum q (ln q - ln p), its derivative to z_j is Q p_j - q_j (a softmax's derivative adds up to zero over a row), and
# distill64 of tests/head_reference.py has p_j - q_j, which adds up to 1 - Q.  The difference (Q - 1) p_j W is three times what
# the float32 paths are allowed; test_lists_above_one and its differences hold the right value.
WRONG_VALUE = {f"test_distillation[f32-{path}-f32-tail-3-8-5-5]" for path in ("simt", "tensor")}


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on a B200)")


def pytest_collection_modifyitems(config, items):
    for item in items:
        if item.name in WRONG_VALUE:
            item.add_marker(pytest.mark.xfail(reason="expects p - q where the loss's derivative is Q p - q", strict=True))
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no CUDA device")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
