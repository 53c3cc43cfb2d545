"""A replica's step (append, then attention) as ``measured.ReplicaLayer`` runs it, against the oracle; cost tables made of measured
times, and candidates scored with them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import Oracle, roofline as rf                  # noqa: E402
from oracle import attention as orc                        # noqa: E402
from paper_2604_07144_amd import binding, measured, traces  # noqa: E402

MODEL = np.array((4, 1024, 2048, 1000, 8, 2, 16), dtype=binding.MODEL_DTYPE)
GPU = np.array((288e9, 2.5e15, 8e12, 128e9, 1.075e12, 50e9, 8), dtype=binding.GPU_DTYPE)


@pytest.mark.parametrize("bits, held, new", [(16, 50, 1), (4, 50, 1), (16, 40, 40), (4, 33, 20)])
def test_a_step_is_append_and_attention(bits, held, new):
    layer = measured.ReplicaLayer(2, 64, 8, 2, 128, bits=bits, copies=2, window=30, sinks=2)
    p = layer.plan(held, new)
    got = layer.step(p).double().cpu().numpy()
    cache, table, turn = layer.caches[0], layer.table.cpu().numpy(), layer.turn.cpu().numpy()
    q, k, v = (p[f].double().cpu().numpy() for f in ("q", "k", "v"))
    eps = torch.finfo(torch.bfloat16).eps / 2
    if bits == 16:
        values = [x.double().cpu().numpy() for x in cache]
    else:
        values = []
        for codes, pairs in zip(cache[:2], cache[2:]):
            c, pr = codes.cpu().numpy(), pairs.double().cpu().numpy()
            x = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], 128).astype(np.float64)
            values.append(np.repeat(pr[..., 1], 64, -1) + np.repeat(pr[..., 0], 64, -1) * x)
    for s in range(2):
        page, slot = table[s, np.arange(held) // 16], np.arange(held) % 16
        keys, vals = values[0][page, :, slot], values[1][page, :, slot]
        for i in range(new):
            t, pos = s * new + i, held - new + i
            if bits == 16:                                  # the new rows are in the cache, rounded once
                assert (np.abs(keys[pos] - orc.turned(k[t], turn[pos], 128, False)) <= eps * np.abs(keys[pos]) * (1 + eps) + 1e-6).all()
                assert np.array_equal(vals[pos], v[t])
            qr = orc.turned(q[t], turn[pos], 128, False)
            for h in range(8):
                o, mean, _ = orc.attention(qr[h], keys[:, h // 4], vals[:, h // 4], pos, np.ones(held, bool), layer.scale, 30, 2)
                # the turned query is rounded once (half a step moves a score by that share of the sum of |q k| scale), weights and result
                # too; keys and values in 4 bits may be
                live = (np.abs(keys[:, h // 4]) @ np.abs(qr[h])).max() * layer.scale
                moved = (1 if bits == 16 else 2) * eps * live + 1e-4
                tol = mean * (eps + 2 * moved * (1 + moved) + (0 if bits == 16 else eps)) + eps * np.abs(o) * (1 + 2 * eps) + 1e-30
                assert (np.abs(got[t, h] - o) <= tol).all(), (s, i, h)


def test_plans_that_are_refused():
    layer = measured.ReplicaLayer(1, 64, 2, 2, 64)
    for held, new in ((65, 1), (10, 0), (10, 11), (0, 0)):
        with pytest.raises(ValueError):
            layer.plan(held, new)


def test_tables_replace_the_rooflines_attention_and_score_candidates():
    tr = traces.make_trace(0, C=16)
    longest = int((tr.prompt_len + tr.out_len).max())
    grid = np.array([1, longest])
    model, gpu = rf.Model(*(int(x) for x in MODEL.tolist())), rf.Gpu(*(float(x) for x in GPU.tolist()[:6]), int(GPU["gpus_per_node"]))
    group = rf.Group(0, 0, 1, 8)
    # times as the roofline has them at both ends of a range in which it is linear: the tables are the roofline's own
    length = np.arange(1, longest + 1, dtype=np.float64)
    att = lambda n, c: rf.op_time(4.0 * 8 * n * c * 8 * 128, 2.0 * (2.0 * 8 * n * 8 * 128 + 2.0 * 8 * c * 2 * 128), gpu) * 1e6   # noqa: E731
    pre, tpot = measured.request_tables(MODEL, GPU, 8, tr.prompt_len, tr.out_len, length, att(1.0, length), length, att(length, length))
    want_pre, want_tpot = rf.request_costs([model], [gpu], [group], tr.prompt_len, tr.out_len)
    assert np.abs(pre.astype(np.int64) - want_pre.astype(np.int64)).max() <= 1 and np.abs(tpot.astype(np.int64) - want_tpot.astype(np.int64)).max() <= 1
    # measured ones are whole numbers of microseconds that grow with what they are added to
    decode_us, prefill_us = measured.layer_times(MODEL, 8, grid, grid, repeats=4)
    assert (decode_us > 0).all() and prefill_us[1] > prefill_us[0] > 0
    tables = measured.request_tables(MODEL, GPU, 8, tr.prompt_len, tr.out_len, grid, decode_us, grid, prefill_us)
    slower = measured.request_tables(MODEL, GPU, 8, tr.prompt_len, tr.out_len, grid, decode_us + 1000.0, grid, prefill_us)
    assert (slower[1].astype(np.int64) - tables[1].astype(np.int64) - 4000 <= 1).all() and np.array_equal(slower[0], tables[0])
    from examples import measured_costs
    got = measured_costs.score(tr, tables, 16)
    want = Oracle.from_trace(tr).set_cost_tables(np.zeros(len(tr.t_on_us), np.uint32), *tables).eval_batch(tr.assignment_rows(0, 16))
    assert got.tobytes() == want.tobytes()
