import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu on the GPU box)")
    config.addinivalue_line("markers", "slow: full-size case, minutes of oracle time")


# A test whose expected value is wrong; it stays as it is.  test_places expects the token of a sequence of 2^31 - 1 tokens at the last place of a table of
# 48, where the contract (include/fobq.h: token t at table entry t / page_size; tokens behind the table are not there) has no page for it.  All
# of its statements, with that one as the contract has it, are in test_lowbit_limits.py.
WRONG = {"test_lowbit_host.py::test_places": "expects a token behind the table at the table's last place"}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG.get(item.nodeid.rsplit("/", 1)[-1])
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, strict=True))
