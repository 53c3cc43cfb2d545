"""Host side of the measured cost tables, no GPU: measurements that are refused (before anything is asked of a device)."""
import numpy as np
import pytest

from paper_2604_07144_amd import binding, measured

MODEL = np.array((4, 1024, 2048, 1000, 8, 2, 16), dtype=binding.MODEL_DTYPE)
GPU = np.array((288e9, 2.5e15, 8e12, 128e9, 1.075e12, 50e9, 8), dtype=binding.GPU_DTYPE)
GOOD = dict(contexts=[16, 64, 149], decode_us=[5.0, 6.0, 7.0], prompts=[16, 100], prefill_us=[8.0, 40.0])
BAD = [dict(contexts=[16, 64, 148]), dict(prompts=[16, 99]), dict(contexts=[64, 16, 149]), dict(prompts=[100, 100]), dict(contexts=[0, 64, 149]), dict(prompts=[100]),
       dict(decode_us=[5.0, 6.0]), dict(prompts=[], prefill_us=[]), dict(prefill_us=[8.0, float("nan")]), dict(decode_us=[5.0, -1.0, 7.0]), dict(contexts=[[16, 64, 149]])]


class Reached(Exception):
    pass


def _tables(monkeypatch, **change):
    def roofline(*args):
        raise Reached

    monkeypatch.setattr(binding, "ap_roofline_tables", roofline)
    return measured.request_tables(MODEL, GPU, 8, [100, 20], [50, 3], **{**GOOD, **change})


@pytest.mark.parametrize("change", BAD)
def test_measurements_that_are_refused(change, monkeypatch):
    """Lengths out of order, shorter than a prompt of 100 or a context of 149, or without their times."""
    with pytest.raises(ValueError):
        _tables(monkeypatch, **change)


def test_lengths_may_end_at_the_longest(monkeypatch):
    with pytest.raises(Reached):
        _tables(monkeypatch)


@pytest.mark.parametrize("weights4", [False, True])
def test_the_example_compares_like_with_like(monkeypatch, capsys, weights4):
    """Times of weights in 4 bits stand beside the roofline of a model whose weights are in 4 bits, and take its terms' places."""
    from examples import measured_costs as example
    bits = []
    monkeypatch.setattr(binding, "ap_workload_create", lambda *a: 1)
    monkeypatch.setattr(binding, "ap_workload_destroy", lambda w: None)
    monkeypatch.setattr(binding, "ap_roofline_costs", lambda w, n, models, gpus, groups: bits.append(int(models[0]["weight_bits"])) or (None, None))
    monkeypatch.setattr(example.measured, "layer_times", lambda model, n, contexts, prompts, **k: bits.append(int(model["weight_bits"])) or (contexts, prompts))
    monkeypatch.setattr(example.measured, "weight_times", lambda model, n, prompts: bits.append(int(model["weight_bits"])) or (1.0, prompts, 1.0))
    monkeypatch.setattr(example.measured, "request_tables", lambda model, *a: bits.append(int(model["weight_bits"])) or (None, None))
    monkeypatch.setattr(example, "score", lambda tr, tables, n: np.ones(n, binding.METRICS_DTYPE))
    assert example.main(["--candidates", "2"] + ["--weights4"] * weights4) == 0
    assert len(bits) == 3 + weights4 and set(bits) == {4 if weights4 else 16}
    assert f"weights in {4 if weights4 else 16} bits" in capsys.readouterr().out
