"""Cost tables made of measured times: what a coarse grid of lengths gives between them, and that every measured time counts."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2604_07144_amd import binding, measured, traces  # noqa: E402

MODEL = np.array((4, 1024, 2048, 1000, 8, 2, 16), dtype=binding.MODEL_DTYPE)
GPU = np.array((288e9, 2.5e15, 8e12, 128e9, 1.075e12, 50e9, 8), dtype=binding.GPU_DTYPE)


@pytest.fixture(scope="module")
def lengths():
    tr = traces.make_trace(0, C=16)
    longest = int((tr.prompt_len + tr.out_len).max())
    return tr.prompt_len, tr.out_len, longest


def _tables(lengths, contexts, decode_us, prompts, prefill_us):
    x = measured.request_tables(MODEL, GPU, 8, lengths[0], lengths[1], contexts, decode_us, prompts, prefill_us)
    return [t.astype(np.int64) for t in x]


def test_curves_between_coarse_lengths(lengths):
    """Times that go as a + b n and a + b n + c n^2, on a grid of powers of two as a user takes it: as if each length had been measured."""
    longest = lengths[2]
    every = np.arange(1, longest + 1)
    coarse = np.unique(np.concatenate([2 ** np.arange(0, int(np.log2(longest)) + 1), [longest]]))
    decode, prefill = lambda n: 20.0 + 0.05 * n, lambda n: 30.0 + 0.2 * n + 0.01 * n * n      # noqa: E731
    want = _tables(lengths, every, decode(every), every, prefill(every))
    got = _tables(lengths, coarse, decode(coarse), coarse, prefill(coarse))
    for w, g in zip(want, got):
        assert np.abs(w - g).max() <= 1                     # whole numbers either way
    assert len(coarse) < len(every) / 16


def test_steps_between_lengths_stay_between_them(lengths):
    """Times with a jump: no time between two lengths lies outside of the two's."""
    grid, us = np.array([1.0, 64, 65, 512, lengths[2]]), np.array([10.0, 10, 50, 50, 60])
    x = measured._between(np.arange(1, lengths[2] + 1, dtype=np.float64), grid, us)
    assert (np.diff(x) >= 0).all() and x[0] == 10 and x[63] == 10 and x[64] == 50 and x[-1] == 60
    assert (measured._between(np.array([1.0, 7.0]), np.array([7.0]), np.array([3.0])) == 3).all()


def test_every_measured_time_counts(lengths):
    """1000 us more at every length are 1000 us for each of the 4 layers: in each step of a request, and in its prefill."""
    grid = np.array([1, 40, 700, lengths[2]])
    decode, prefill = np.array([20.0, 25.0, 90.0, 300.0]), np.array([30.0, 60.0, 5000.0, 90000.0])
    base = _tables(lengths, grid, decode, grid, prefill)
    slow_step, slow_start = _tables(lengths, grid, decode + 1000, grid, prefill), _tables(lengths, grid, decode, grid, prefill + 1000)
    assert np.abs(slow_step[1] - base[1] - 4000).max() <= 1 and np.array_equal(slow_step[0], base[0])
    assert np.abs(slow_start[0] - base[0] - 4000).max() <= 1 and np.array_equal(slow_start[1], base[1])
