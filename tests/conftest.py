import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run with -m gpu on a B200)")


def pytest_collection_modifyitems(config, items):
    """Skip GPU tests when no device is present, so a plain `pytest tests` stays green on CPU."""
    try:
        import torch
        have_gpu = torch.cuda.is_available()
    except Exception:
        have_gpu = False
    if have_gpu:
        return
    skip = pytest.mark.skip(reason="no CUDA device")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)


@pytest.fixture(autouse=True, scope="session")
def garbage_goes_before_a_capture():
    """A CUDA graph that garbage collection destroys while another is captured ends that capture (error 901), and a test that has looked into an exception leaves its frame, with the
    graphs in it, to the collector: it runs before every capture."""
    import gc
    try:
        import torch
        if not torch.cuda.is_available():
            raise ImportError
    except ImportError:
        yield
        return
    enter = torch.cuda.graph.__enter__

    def collected(self):
        gc.collect()
        return enter(self)
    torch.cuda.graph.__enter__ = collected
    yield
    torch.cuda.graph.__enter__ = enter
