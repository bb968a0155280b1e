import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long CPU test")


def gpu_available() -> bool:
    try:
        import torch
        return bool(torch.cuda.is_available())
    except Exception:
        return False


@pytest.fixture(scope="session", autouse=True)
def streams_in_use():
    """Work on as many streams as a process has hardware queues, before any test: the first use of a queue holds up the other
    streams' work for milliseconds (6.5 ms measured), in which a fill on one stream and a kernel on another change places."""
    if not gpu_available():
        return
    import torch
    x = torch.zeros(64, device="cuda")
    for _ in range(8):
        with torch.cuda.stream(torch.cuda.Stream()):
            x + 1
        torch.cuda.synchronize()


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")
