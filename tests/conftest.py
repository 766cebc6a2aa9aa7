import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (B200); run with -m gpu")


@pytest.fixture(autouse=True)
def operators_are_bound_again():
    """A test may bind the compiled Python calls, which all tests share, to entries, a device and a stream of its own; the next
    operator call binds them to the library again."""
    yield
    binding = sys.modules.get("paper_2511_04063_b200.binding")
    if binding is not None:
        binding._calls = None


@pytest.fixture(scope="session")
def dq():
    """The Python binding over the C-ABI library (GPU tests only)."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2511_04063_b200 as pkg
    return pkg
