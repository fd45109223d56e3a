import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on the B200 box)")


def pytest_collection_modifyitems(config, items):
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


@pytest.fixture(autouse=True)
def garbage_is_collected_between_gpu_tests(request):
    """A CUDA graph that Python's garbage collector destroys while another is being captured invalidates that capture: what an
    earlier test has left in cycles (an exception's traceback is enough) would end a later one, depending on the number of
    objects made since."""
    if "gpu" not in request.keywords:
        yield
        return
    gc.collect()
    gc.freeze()        # (what is left lives on: the next collection need not look at it)
    gc.disable()
    yield
    gc.enable()
