"""What ``measured.ReplicaLayer`` times."""
import time

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2604_07144_amd import binding, measured         # noqa: E402


def test_a_slow_host_is_not_in_the_time(monkeypatch):
    """Calls that take the host 2 ms each: a step's time is the device's all the same."""
    layer = measured.ReplicaLayer(2, 64, 8, 2, 128)
    fast, calls = layer.time_us(50, 1, repeats=10), []
    attention = binding.ap_attention

    def slow(*args):
        calls.append(1)
        time.sleep(0.002)
        attention(*args)

    monkeypatch.setattr(binding, "ap_attention", slow)
    us = layer.time_us(50, 1, repeats=10)
    assert len(calls) >= 10 and 0 < fast < 1000 and 0 < us < 1000
