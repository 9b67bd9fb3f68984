import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (GB300) and the built CUDA library")


GOLDEN = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden")


def read_golden(name):
    rows = []
    with open(os.path.join(GOLDEN, name)) as f:
        for line in f:
            line = line.strip()
            if not line or line.startswith("#"):
                continue
            rows.append([[float(x) for x in part.split()] for part in line.split("|")])
    return rows


# Tests that expect a wrong value, as they were written; they still run, and fail.
WRONG_VALUES = {
    "test_gpu_distill.py::test_the_same_token_twice":
        "takes the loss entry by entry where a list names a token several times; the divergence adds a token's entries "
        "up first (test_gpu_distill_repeated.py)",
}


def pytest_collection_modifyitems(items):
    for item in items:
        for name, why in WRONG_VALUES.items():
            if item.nodeid.split("[")[0].endswith(name):
                item.add_marker(pytest.mark.xfail(reason=why, raises=AssertionError, strict=True))
