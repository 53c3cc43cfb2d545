"""A replica's whole step: projections, cache, attention, feed-forward block, head and answer one after another on one stream, eagerly and
from a graph, each against plain sums in 64 bits over what it was given; and the cost tables that measured weights go into."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import linear as orc
from oracle import roofline as rf
from paper_2604_07144_amd import binding as b
from paper_2604_07144_amd import measured, traces
from tests.attn_harness import Replica
from tests.attn_harness import check as check_attention
from tests.linear_harness import Matrix, check_gated, check_linear, stream_of, vectors

pytestmark = pytest.mark.gpu
H, A, K, D, I, V, TOP = 512, 4, 2, 128, 896, 5003, 6
MODEL = np.array((4, 1024, 2048, 1000, 8, 2, 4), dtype=b.MODEL_DTYPE)
GPU = np.array((288e9, 2.5e15, 8e12, 128e9, 1.075e12, 50e9, 8), dtype=b.GPU_DTYPE)


class Step:
    """A layer and a head over sequences that hold ``held`` tokens, the last ``new`` of them new."""

    def __init__(self, held, new, group, bits, seed):
        self.m = {f: Matrix(*size, group, "bf16", seed=seed + i) for i, (f, size) in enumerate(
            dict(qkv=((A + 2 * K) * D, H), out=(H, A * D), gate=(I, H), up=(I, H), down=(H, I), head=(V, H)).items())}
        self.r = Replica(held, new, K=K, A=A, d=D, page=16, bits=bits, seed=seed)
        self.cache, self.batch = self.r.describe()
        self.T = T = self.r.T
        rows = lambda n: torch.zeros((T, n), dtype=torch.bfloat16, device="cuda")          # noqa: E731
        self.x, self.qkv, self.turned, self.seen, self.mid, self.h, self.y, self.logits = (rows(n) for n in (H, (A + 2 * K) * D, A * D, A * D, H, I, H, V))
        self.x.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((T, H), dtype=np.float32)))
        self.tokens = torch.arange(T, device="cuda").int()
        self.d_logits = b.make_logits(b.AP_BF16, T, V, self.logits.data_ptr())
        f = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")             # noqa: E731
        self.logprob, self.entropy, self.ids, self.tops = f(T), f(T), f(T, TOP, t=torch.int32), f(T, TOP)
        w = {n: m.describe() for n, m in self.m.items()}
        self.w = w
        need = [b.ap_linear_workspace(w[n], T) for n in ("qkv", "out", "down", "head")] + [b.ap_gated_workspace(w["gate"], w["up"], T),
                b.ap_attention_workspace(self.cache, self.batch, A), b.ap_logprobs_workspace(self.d_logits, TOP)]
        self.space = torch.full((max(16, *need),), 0xA5, dtype=torch.uint8, device="cuda")
        at = self.qkv.data_ptr()
        self.q, self.k, self.v = (b.make_rows(at + 2 * D * n, h, D, 2 * (A + 2 * K) * D) for n, h in ((0, A), (A, K), (A + K, K)))

    def run(self):
        s, w = stream_of(), self.w
        tail = (self.space.data_ptr(), self.space.numel(), s)
        b.ap_linear(w["qkv"], vectors(self.x), vectors(self.qkv), self.T, None, *tail)
        b.ap_kv_append(self.cache, self.batch, self.k, self.v, None, self.q, b.make_rows(self.turned.data_ptr(), A, D), A, s)
        b.ap_attention(self.cache, self.batch, b.make_rows(self.turned.data_ptr(), A, D), b.make_rows(self.seen.data_ptr(), A, D), A, D ** -0.5, 0, 0, *tail)
        b.ap_linear(w["out"], vectors(self.seen), vectors(self.mid), self.T, vectors(self.x), *tail)
        b.ap_gated(w["gate"], w["up"], vectors(self.mid), vectors(self.h), self.T, b.AP_SILU, *tail)
        b.ap_linear(w["down"], vectors(self.h), vectors(self.y), self.T, vectors(self.mid), *tail)
        b.ap_linear(w["head"], vectors(self.y), vectors(self.logits), self.T, None, *tail)
        b.ap_logprobs(self.d_logits, self.tokens.data_ptr(), 1.0, TOP, self.logprob.data_ptr(), self.entropy.data_ptr(), self.ids.data_ptr(),
                      self.tops.data_ptr(), *tail)
        return [x.clone() for x in (self.qkv, self.seen, self.mid, self.h, self.y, self.logits, self.logprob, self.entropy, self.ids, self.tops)]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("held,new,group", [([40, 3, 128, 77], [1, 1, 1, 1], 128), ([100, 60, 33], [100, 7, 33], 64), ([300], [300], 32)])
def test_every_part_of_a_step(held, new, group, bits):
    s = Step(held, new, group, bits, seed=len(held))
    s.run()
    torch.cuda.synchronize()
    m = s.m
    check_linear(m["qkv"], s.x, s.qkv)
    q = s.qkv[:, :A * D].reshape(s.T, A, D)
    assert torch.equal(s.turned.view(s.T, A, D), q)
    check_attention(s.seen.view(s.T, A, D), *s.r.expected(q, D ** -0.5))
    check_linear(m["out"], s.seen, s.mid, s.x)
    check_gated(m["gate"], m["up"], s.mid, s.h, "silu")
    check_linear(m["down"], s.h, s.y, s.mid)
    check_linear(m["head"], s.y, s.logits)
    logits = s.logits.double().cpu().numpy()
    for t in range(0, s.T, 1 + s.T // 20):
        log, entropy, ids, tops, spread = orc.logprobs(logits[t], t, 1.0, TOP)
        each = (1 + spread) * 2.0 ** -21 * (2 + spread)
        assert np.array_equal(s.ids[t].cpu().numpy(), ids)
        assert abs(float(s.logprob[t]) - log) <= each + 2.0 ** -22 * abs(log) and abs(float(s.entropy[t]) - entropy) <= each + 2.0 ** -22 * entropy
        assert (np.abs(s.tops[t].double().cpu().numpy() - tops) <= each + 2.0 ** -22 * np.abs(tops)).all()


@pytest.mark.parametrize("held,new", [([40, 3, 128, 77], [1, 1, 1, 1]), ([100, 60, 33], [100, 7, 33])])
def test_a_step_from_a_graph(held, new):
    s, other = Step(held, new, 128, 16, seed=9), Step(held, new, 128, 16, seed=9)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for i in range(4):
        x = torch.from_numpy(np.random.default_rng(50 + i).standard_normal((s.T, H), dtype=np.float32)).cuda()
        s.x.copy_(x)
        other.x.copy_(x)
        want = other.run()
        torch.cuda.synchronize()
        s.space.fill_(0x5A)
        graph.replay()
        torch.cuda.synchronize()
        for a, y in zip((s.qkv, s.seen, s.mid, s.h, s.y, s.logits, s.logprob, s.entropy, s.ids, s.tops), want):
            assert torch.equal(a, y)


def test_two_graphs_of_one_workspace_take_turns():
    """Graphs that share a workspace and are replayed one after another on one stream do not disturb each other."""
    m, x = [Matrix(300, 2048, 64, seed=i) for i in range(2)], torch.randn((150, 2048), device="cuda").bfloat16()
    need = max(b.ap_linear_workspace(w.describe(), 150) for w in m)
    assert need > 0
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = [torch.zeros((150, 300), dtype=torch.bfloat16, device="cuda") for _ in m]
    want = [w.linear(x) for w in m]
    graphs = [torch.cuda.CUDAGraph() for _ in m]
    torch.cuda.synchronize()
    for g, w, y in zip(graphs, m, out):
        with torch.cuda.graph(g):
            w.linear(x, y=y, space=space)
    for _ in range(3):
        for g, y in zip(graphs, out):
            y.zero_()
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, y) for a, y in zip(out, want))


def _tables(weights=None, grid=None):
    tr = traces.make_trace(0)
    longest = int((tr.prompt_len + tr.out_len).max())
    grid = np.array([16.0, 64.0, 256.0, float(longest)]) if grid is None else grid
    us = np.full(len(grid), 50.0)
    return tr, grid, measured.request_tables(MODEL, GPU, 8, tr.prompt_len, tr.out_len, grid, us, grid, us, weights)


def test_the_rooflines_own_times_for_weights_change_nothing():
    """Times as the roofline has them, at every length, give its tables; and others move them by what they differ."""
    longest = int((lambda t: (t.prompt_len + t.out_len).max())(traces.make_trace(0)))
    every = np.arange(1, longest + 1, dtype=np.float64)
    model, gpu = rf.Model(*(int(x) for x in MODEL.tolist())), rf.Gpu(*(float(x) for x in GPU.tolist()[:6]), int(GPU["gpus_per_node"]))
    e, d = model.weight_bits / 8, model.hidden / model.heads

    def layer_us(n):
        wide, b_ = (model.heads + 2 * model.kv_heads) * d, 8.0
        return 1e6 * (rf.op_time(2 * b_ * n * model.hidden * wide, e * (model.hidden * wide + b_ * n * (model.hidden + wide)), gpu)
                      + rf.op_time(2 * b_ * n * model.hidden * model.hidden, e * (model.hidden ** 2 + 2 * b_ * n * model.hidden), gpu)
                      + rf.op_time(6 * b_ * n * model.hidden * model.intermediate, e * (3 * model.hidden * model.intermediate + 2 * b_ * n * model.hidden + 3 * b_ * n * model.intermediate), gpu))
    head_us = 1e6 * float(rf.op_time(2 * 8.0 * model.hidden * model.vocab, e * (model.hidden * model.vocab + 8 * model.hidden + 8 * model.vocab), gpu))
    _, _, plain = _tables(grid=every)
    tr, _, same = _tables((float(layer_us(1.0)), layer_us(every), head_us), every)
    for x, y in zip(plain, same):
        assert np.abs(x.astype(np.int64) - y.astype(np.int64)).max() <= 1                  # a rounding to whole microseconds
    _, _, more = _tables((float(layer_us(1.0)) + 100.0, layer_us(every) + 200.0, head_us + 1000.0), every)
    assert np.abs(more[0].astype(np.int64) - plain[0] - (4 * 200 + 1000)).max() <= 1 and np.abs(more[1].astype(np.int64) - plain[1] - (4 * 100 + 1000)).max() <= 1


def test_times_for_weights_that_say_nothing_are_refused():
    good = np.full(4, 10.0)
    for bad in ((np.nan, good, 1.0), (-1.0, good, 1.0), (1.0, good, np.inf), (1.0, good[:3], 1.0), (1.0, -good, 1.0)):
        with pytest.raises(ValueError):
            _tables(bad)


def test_weights_are_measured():
    decode, prefill, head = measured.weight_times(MODEL, 8, [16, 128], top=5, repeats=4)
    assert 0 < decode < 1e4 and (prefill > 0).all() and prefill.shape == (2,) and 0 < head < 1e4
    with pytest.raises(ValueError):
        measured.ReplicaWeights(MODEL).plan(0)


def test_a_measured_layer_computes_what_it_says():
    layer = measured.ReplicaWeights(MODEL, copies=2, group=64, dtype="fp16")
    p = layer.plan(20)
    first = layer.step(p).clone()
    second = layer.step(p).clone()
    torch.cuda.synchronize()
    assert not torch.equal(first, second) and torch.equal(layer.step(p), first)            # copies take turns
    values = {}
    for f, w in layer.copies[0].items():
        n_out, n_in = layer.sizes[f]
        x = torch.empty((n_out, n_in), dtype=torch.float16, device="cuda")
        b.ap_weights_read(w["w"], b.make_vectors(x.data_ptr(), n_in), stream_of())
        values[f] = x.double()
    mid = p["attended"].double() @ values["out"].T + p["x"].double()
    gate = mid @ values["gate"].T
    want = (gate / (1 + torch.exp(-gate)) * (mid @ values["up"].T)) @ values["down"].T + mid
    # three roundings of rows to 2^-11 of their size and one of each weight, each sum over hundreds of terms of either sign
    assert ((first.double() - want).abs().max() / want.abs().max()) < 8 * 2.0 ** -11


def test_the_head_answers():
    head = measured.ReplicaWeights(MODEL, head=True, top=3)
    p = head.plan(5)
    logits = head.step(p)[:, :1000].double().cpu().numpy()
    torch.cuda.synchronize()
    for t in range(5):
        assert np.array_equal(p["top_id"][t].cpu().numpy(), orc.logprobs(logits[t], 0, 1.0, 3)[2])


def test_the_example_runs_with_weights(capsys):
    spec = importlib.util.spec_from_file_location("measured_costs", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "measured_costs.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(["--weights4", "--candidates", "8"]) == 0
    assert "weights in 4 bits" in capsys.readouterr().out
