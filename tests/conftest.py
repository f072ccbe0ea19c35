import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu on the GPU box)")


@pytest.fixture(autouse=True)
def library_choices():
    """A test that fails with knobs set leaves none of them to the next."""
    yield
    ssd = sys.modules.get("paper_2603_09555_amd.ssd")
    if ssd is not None:
        ssd.reset_knobs()


def pytest_collection_modifyitems(config, items):
    # GPU tests are skipped (not failed) where no device exists, so a plain `pytest tests/` works anywhere.
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover
        has_gpu = False
    if has_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU in this container")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
