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


@pytest.fixture
def fills_end(monkeypatch):
    """torch.zeros_like whose fill has ended when it returns."""
    import torch
    zeros_like = torch.zeros_like

    def filled(*args, **kw):
        t = zeros_like(*args, **kw)
        torch.cuda.synchronize()
        return t
    monkeypatch.setattr(torch, "zeros_like", filled)


def pytest_collection_modifyitems(items):
    # This test fills its output on the current stream after the other stream has waited for that one: nothing else orders the fill
    # before the attention that writes there (the first use of a hardware queue held a fill up by 6.5 ms).
    for item in items:
        if item.nodeid.endswith("test_gpu_kv8.py::test_another_stream"):
            item.fixturenames.append("fills_end")


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")
