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
    go to them in turn as each is first used, the default stream's among them.  The module leaves whole rounds of used
    streams, so that tests after it, some of which keep the default stream busy, meet the queues that they would have
    met without it."""
    yield
    import torch
    if not torch.cuda.is_available():
        return
    for _ in range(4):
        s = torch.cuda.Stream()
        if (s.stream_id >> 5) % 4 == 3:
            break
    for i in range((s.stream_id >> 5) + 1):
        with torch.cuda.stream(torch.cuda.Stream(stream_id=s.stream_id & 31 | i << 5, device_index=s.device_index,
                                                 device_type=s.device_type)):
            torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
