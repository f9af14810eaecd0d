import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: longer CPU-only test")


# Unmarked tests with a call that passes every host check with invented pointers: where a GPU
# is, its kernel would run on them.  (What it checks there is checked on the stand-in runtime by
# test_f8.py's test_append_takes_pages_of_one_request_each.)
INVENTED_POINTERS = ("test_f8.py::test_append_refuses_a_page_of_two_requests",)


def kept_from_a_gpu(nodeid, gpu=None):
    gpu = os.path.exists("/dev/kfd") if gpu is None else gpu
    return gpu and nodeid.split("[")[0].endswith(INVENTED_POINTERS)


def pytest_runtest_setup(item):
    if kept_from_a_gpu(item.nodeid):
        pytest.skip("launches with invented pointers where a GPU is")
