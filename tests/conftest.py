"""Shared pytest configuration: the ``gpu`` marker and common fixtures."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


# Tests that assert what the documentation rules out; others hold what is right in their place.
WRONG = {
    "test_decode_step_gpu.py::test_pages_that_are_none":
        "adds weights through a table entry that names no page to page 0, never written through by include/fqvit.h; "
        "test_decode_pages.py has its calls with the right weights",
}


def pytest_collection_modifyitems(items):
    for item in items:
        for name, why in WRONG.items():
            if item.nodeid.endswith(name):
                item.add_marker(pytest.mark.xfail(reason=why, raises=AssertionError, strict=True))


@pytest.fixture(scope="session")
def orc():
    """The CPU oracle (built on first use)."""
    import oracle
    oracle.build(force=False)
    return oracle


@pytest.fixture(scope="session")
def plan(tmp_path_factory):
    """What a Log-Int-Softmax call launches (tests/launch_plan.py)."""
    from launch_plan import Launches
    return Launches(tmp_path_factory.mktemp("plan"))
