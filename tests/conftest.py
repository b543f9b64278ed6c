import os
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (runs the hand-written kernels through the C ABI)")


def pytest_collection_modifyitems(config, items):
    # A GPU test on a machine without one is a skip, never a silent CPU fallback.
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if not has_gpu:
        skip = pytest.mark.skip(reason="no CUDA device")
        for it in items:
            if "gpu" in it.keywords:
                it.add_marker(skip)


@pytest.fixture(autouse=True)
def _collect_after_gpu_test(request):
    """A test that catches an error keeps its frame, and with it a context's device buffers, alive in a reference cycle.
    They go with the test, not whenever the collector next runs -- which may be between two readings of the allocator in
    a later one."""
    yield
    if "gpu" in request.node.keywords:
        import gc
        gc.collect()


@pytest.fixture(scope="session", autouse=True)
def _what_takes_its_time_once(request):
    """What takes its time once: memory for a stream of torch's pool (its allocator asks the driver: 0.4 ms, but 20 to 100 where other users
    of the machine allocate) and loading a library's kernel (zeros 8 ms).  Done ahead of tests that count on what a stream of theirs is
    still doing (10 ms of sleep); a block of every stream is held, since a capture empties the cache."""
    import torch
    blocks = []
    if torch.cuda.is_available() and any("gpu" in it.keywords for it in request.session.items):
        torch.cuda._sleep(1)
        torch.zeros((64, 1024), device="cuda")
        for stream in [torch.cuda.Stream() for _ in range(32)]:              # (the pool's, in turn)
            with torch.cuda.stream(stream):
                blocks.append(torch.empty(1, device="cuda"))
        torch.cuda.synchronize()
    yield
    blocks.clear()
