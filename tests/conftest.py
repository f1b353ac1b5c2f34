import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built libmalt")
    config.addinivalue_line("markers", "slow: long-running (full-size) case")


@pytest.fixture(scope="module")
def stream_rounds():
    """For a module that takes streams: torch hands them out of a pool in turn, and the card's four hardware queues
    are behind them in turn, the default stream's among them.  The pool is left where a round starts, so that tests
    after the module, some of which keep the default stream busy, meet the queues that they would have met without it."""
    yield
    import torch
    if torch.cuda.is_available():
        for _ in range(4):
            if (torch.cuda.Stream().stream_id >> 5) % 4 == 3:
                break
