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


def _pages(layer, batch):
    """The (sequence's) pages that a step's description names."""
    at = (batch.page_table - layer.table.data_ptr()) // 4
    return layer.table.view(-1)[at:at + (batch.n_seqs - 1) * batch.table_stride + batch.table_width].cpu().as_strided((batch.n_seqs, batch.table_width), (batch.table_stride, 1))


def test_timed_steps_come_back_to_their_pages_late(monkeypatch):
    """Between two steps over the same pages more is read than the chip's caches hold, at short lengths as at the longest."""
    seen, model = [], np.array((32, 4096, 14336, 128256, 32, 8, 16), dtype=binding.MODEL_DTYPE)
    attention, time_us = binding.ap_attention, measured.ReplicaLayer.time_us

    def logged(cache, batch, *args):
        seen[-1][2].append((cache.k, batch.page_table, batch.table_width, batch.max_kv))
        seen[-1][3] = (cache, batch)
        attention(cache, batch, *args)

    def timed(layer, held, new, repeats):
        seen.append([layer, held, [], None])
        return time_us(layer, held, new, repeats)

    monkeypatch.setattr(binding, "ap_attention", logged)
    monkeypatch.setattr(measured.ReplicaLayer, "time_us", timed)
    measured.layer_times(model, 8, [64, 700, 8192, 32768], [64], repeats=40)
    assert [x[1] for x in seen] == [64, 700, 8192, 32768, 64]
    for layer, held, calls, (cache, batch) in seen:
        size = 2 * 8 * held * 8 * 2 * 128                   # bytes of keys and values that a step reads
        last, taken = {}, {}
        for i, (k, table, width, max_kv) in enumerate(calls):
            assert width * layer.page >= max_kv == held
            if (k, table) in last:
                assert (i - last[k, table]) * size > 1 << 28, held
            last[k, table] = i
            batch.page_table = table
            pages = _pages(layer, batch)
            assert pages.unique().numel() == pages.numel()
            taken.setdefault(k, {})[table] = set(pages.flatten().tolist())
        for tables in taken.values():                       # no page in two turns of a cache
            assert sum(len(x) for x in tables.values()) == len(set().union(*tables.values()))


@pytest.mark.parametrize("bits", [16, 4])
def test_every_turn_is_a_step_over_its_own_pages(bits):
    """Each turn's new rows are on its own pages, and what it gives is what the same rows give on any pages of the same content."""
    layer = measured.ReplicaLayer(3, 256, 8, 2, 128, bits=bits, copies=2)
    p = layer.plan(100, 5)
    cache = layer.caches[0]
    assert len(p["turns"]) == 2 * (256 // 16 // 7)
    for x in cache:                                         # the next pages get the first ones' content
        x[layer.table[:, 7:14].long().flatten()] = x[layer.table[:, :7].long().flatten()]
    outs = [layer.step(p).clone() for _ in range(4)]
    assert torch.equal(outs[0], outs[2]) and not torch.equal(outs[0], outs[1])   # turns go cache by cache, then on to the next pages
    for x in cache:
        assert torch.equal(x[layer.table[:, :7].long()], x[layer.table[:, 7:14].long()])
    if bits == 16:
        rows = cache[1][layer.table[:, 7 + 99 // 16].long(), :, 99 % 16]
        assert torch.equal(rows, p["v"].view(3, 5, 2, 128)[:, 4])


def test_calls_are_made_with_the_layers_device_as_the_present_one(monkeypatch):
    """Kernels go to the present device, so a layer of another one makes it that for its calls."""
    layer, active, devices = measured.ReplicaLayer(1, 64, 2, 2, 64, device="cuda:0"), [], []
    real, append, attention = torch.cuda.device, binding.ap_kv_append, binding.ap_attention

    class Guard(real):
        def __enter__(self):
            active.append(self.idx)
            return super().__enter__()

        def __exit__(self, *args):
            active.pop()
            return super().__exit__(*args)

    def logged(call):
        return lambda *args: (devices.append(active[-1] if active else None), call(*args))

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(binding, "ap_kv_append", logged(append))
    monkeypatch.setattr(binding, "ap_attention", logged(attention))
    layer.step(layer.plan(20, 1))
    layer.time_us(20, 1, repeats=2)
    assert len(devices) >= 4 and set(devices) == {0} and not active


@pytest.mark.parametrize("batch, longest", [(1, 16), (8, 64), (64, 300)])
def test_short_models_do_not_make_more_caches_than_steps(batch, longest, monkeypatch):
    """Where a cache is small, as many turns as there are steps in a timing do: the chip's caches hold other memory when it begins."""
    model, made, steps = np.array((4, 256, 2048, 1000, 4, 1, 16), dtype=binding.MODEL_DTYPE), [], []
    init, attention = measured.ReplicaLayer.__init__, binding.ap_attention

    def logged(layer, *args, **kw):
        init(layer, *args, **kw)
        made.append(layer)

    def call(cache, batch, *args):
        steps.append((cache.k, batch.page_table))
        attention(cache, batch, *args)

    monkeypatch.setattr(measured.ReplicaLayer, "__init__", logged)
    monkeypatch.setattr(binding, "ap_attention", call)
    decode_us, prefill_us = measured.layer_times(model, batch, [longest], [longest], repeats=12)
    assert decode_us[0] > 0 and prefill_us[0] > 0 and 1 <= len(made[0].caches) <= 12
    recorded = steps[1:13]                                  # after the first step, the decode steps of the graph
    assert len(set(recorded)) == 12
