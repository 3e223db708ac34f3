import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


@pytest.fixture(autouse=True)
def _made_up_addresses_reach_no_gpu(request, monkeypatch):
    """tests/test_abi_cpu.py passes made-up addresses and counts on there being no GPU. Where there is one, its
    accepted calls end right before the launch."""
    if request.module.__name__.rpartition(".")[2] == "test_abi_cpu":
        import torch
        if torch.cuda.device_count() > 0:
            monkeypatch.setenv("RELATION_TEST_FAIL_LAUNCH", "1")
