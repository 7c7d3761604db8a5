import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (runs through the C-ABI on the GPU)")


# Tests that hold a wrong value, and why it is; each has a counterpart with the right one.
WRONG = {
    "test_gpu_paged.py::test_tables_keep_more_than_there_is":
        "a slot that was given 40 tokens keeps 40, not the 64 that its pages have room for "
        "(test_gpu_paged_dry_pool.py::test_keep_more_than_there_is)",
}


def pytest_collection_modifyitems(items):
    for item in items:
        for name, why in WRONG.items():
            if item.nodeid.endswith(name):
                item.add_marker(pytest.mark.xfail(reason=why, strict=True))


def pytest_sessionfinish(session, exitstatus):
    """Keep the parity runs' largest attention errors (and their fraction of
    the tolerance) as JSON when any ran: at BATON_MARGINS_OUT, else as
    parity_margins.json in the results folder the GPU runs hand back."""
    parity = sys.modules.get("tests.parity")
    if parity is not None:
        parity.write_margins(os.environ.get("BATON_MARGINS_OUT",
                                            os.path.join(ROOT, "gpurun_out", "parity_margins.json")))
