"""Cost tables with a replica's step measured on the card.

The roofline prices every operator of a model analytically.  What goes by the lengths in a trace is the cache of keys and
values and the attention over it; this module runs those (``ap_kv_append``, ``ap_attention``) on the present device at a grid of
lengths and puts the measured times in the place of the roofline's attention term, so that ``ap_costtable_set`` can score
candidates with them.  For replicas whose weights are held in 4 bits the projections and feed-forward blocks (``ap_linear``,
``ap_gated``) and the output head with its answer (``ap_linear``, ``ap_logprobs``) can be measured alike; what is not stays the
roofline's, as the all-reduce does.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding

CHIP_CACHE = 256 << 20                  # bytes: the largest of the card's caches
DTYPES = {"bf16": (torch.bfloat16, binding.AP_BF16), "fp16": (torch.float16, binding.AP_FP16)}


class ReplicaLayer:
    """One layer's cache of a replica: ``batch`` slots of up to ``max_len`` tokens in shuffled pages, and a step over them.

    ``heads``, ``kv_heads`` and ``head_dim`` are the layer's; ``bits`` is what the cache is held in (16 or 4).  There are caches of
    ``copies`` layers.  Steps of fewer than ``max_len`` tokens take turns at the pages that a slot has, then at the caches, so that each of
    them comes back to its pages only after all the others, as a layer of a served model does."""

    def __init__(self, batch: int, max_len: int, heads: int, kv_heads: int, head_dim: int, *, dtype: str = "bf16", bits: int = 16,
                 page: int = 16, copies: int = 1, window: int = 0, sinks: int = 0, device: str = "cuda", seed: int = 0):
        self.batch, self.max_len, self.heads, self.kv_heads, self.head_dim = batch, max_len, heads, kv_heads, head_dim
        self.torch_dtype, self.dtype = DTYPES[dtype]
        self.bits, self.page, self.window, self.sinks = bits, page, window, sinks
        self.device = device = torch.empty(0, device=device).device    # with its number
        self.scale = head_dim ** -0.5
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        width = -(-max_len // page)
        self.n_pages = batch * width
        self.table = torch.randperm(self.n_pages, generator=gen, device=device).int().view(batch, width)
        row = (self.n_pages, kv_heads, page)
        self.caches = []
        for _ in range(copies):
            if bits == 16:
                self.caches.append([torch.randn((*row, head_dim), generator=gen, device=device).to(self.torch_dtype) for _ in range(2)])
            else:
                codes = [torch.randint(0, 256, (*row, head_dim // 2), generator=gen, device=device, dtype=torch.uint8) for _ in range(2)]
                pairs = torch.tensor([0.25, -1.875], device=device).to(self.torch_dtype)        # step and lowest value
                self.caches.append(codes + [pairs.repeat(*row, head_dim // 64, 1).contiguous() for _ in range(2)])
        angle = torch.arange(max_len, device=device, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float64) / head_dim)
        self.turn = torch.stack([angle.cos(), angle.sin()], -1).float()
        self.gen = gen

    def plan(self, held: int, new: int) -> dict:
        """Memory and descriptions of steps in which every slot holds ``held`` tokens, ``new`` of them new: ``turns`` of them, a cache and
        its pages each.  The first one's pages are the first of each slot."""
        if not 1 <= new <= held <= self.max_len:
            raise ValueError(f"a step of {new} new tokens of {held} in slots of {self.max_len}")
        b, T, made = self.batch, self.batch * new, lambda h: torch.randn((self.batch * new, h, self.head_dim), generator=self.gen, device=self.device).to(self.torch_dtype)
        p = dict(first=(torch.arange(b + 1, device=self.device) * new).int(), held=torch.full((b,), held, dtype=torch.int32, device=self.device),
                 q=made(self.heads), k=made(self.kv_heads), v=made(self.kv_heads))
        p["turned"], p["out"] = torch.empty_like(p["q"]), torch.empty_like(p["q"])
        p["rows"] = {f: binding.make_rows(p[f].data_ptr(), p[f].shape[1], self.head_dim) for f in ("q", "k", "v", "turned", "out")}
        width, pages = self.table.shape[1], -(-held // self.page)
        batches = [binding.make_seq_batch(b, T, new, held, p["first"].data_ptr(), p["held"].data_ptr(), self.table.data_ptr() + 4 * at, pages, width)
                   for at in range(0, width - pages + 1, pages)]
        caches = [binding.make_kv_cache(self.dtype, self.bits, self.n_pages, self.page, self.kv_heads, self.head_dim, *(x.data_ptr() for x in c))
                  for c in self.caches]
        p["at"], p["turns"] = 0, [(c, x) for x in batches for c in caches]
        p["rotation"] = binding.make_rotation(self.turn.data_ptr(), self.max_len, self.head_dim)
        p["space"] = torch.empty(max(16, binding.ap_attention_workspace(caches[0], batches[0], self.heads, self.window, self.sinks)),
                                 dtype=torch.uint8, device=self.device)
        return p

    def step(self, p: dict) -> torch.Tensor:
        """The new tokens into the cache, turned, and their attention over it: [token][head][channel]."""
        (cache, batch), rows = p["turns"][p["at"]], p["rows"]
        p["at"] = (p["at"] + 1) % len(p["turns"])
        with torch.cuda.device(self.device):                # kernels go to the device that is the present one
            stream = torch.cuda.current_stream().cuda_stream
            binding.ap_kv_append(cache, batch, rows["k"], rows["v"], p["rotation"], rows["q"], rows["turned"], self.heads, stream)
            binding.ap_attention(cache, batch, rows["turned"], rows["out"], self.heads, self.scale, self.window, self.sinks,
                                 p["space"].data_ptr(), p["space"].numel(), stream)
        return p["out"]

    def time_us(self, held: int, new: int, repeats: int = 20) -> float:
        """Microseconds of a step among others: the median of five timings of ``repeats`` steps each.  The steps are recorded into a graph,
        so that the device's time is taken and not that of the host's calls; before each timing the caches of the chip are filled with
        other memory."""
        with torch.cuda.device(self.device):
            p = self.plan(held, new)
            return _graph_us(lambda: self.step(p), repeats, self.device)


def _graph_us(step, repeats: int, device) -> float:
    """Median of five timings of ``repeats`` steps in a graph, microseconds a step; other memory fills the chip's caches before each."""
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(repeats):
            step()
    other, times = torch.zeros(2 * CHIP_CACHE // 4, dtype=torch.int32, device=device), []
    graph.replay()
    for _ in range(5):
        a, z = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        other.sum()                                     # also keeps the device busy until what is timed has been sent
        a.record()
        graph.replay()
        z.record()
        z.synchronize()
        times.append(a.elapsed_time(z) * 1e3 / repeats)
    return float(np.median(times))


class ReplicaWeights:
    """Matrices of a model in 4 bits, ``copies`` times, and steps of ``n_tokens`` rows through them: a layer's projections and
    feed-forward block (``layer``), or the output head with the log probabilities of its ``top`` alternatives (``head``).

    ``model`` is a record of ``binding.MODEL_DTYPE``; ``group`` columns share a pair.  The values are random, which no time depends on.
    Steps take turns at the copies, so that each comes back to its weights only after all the others."""

    def __init__(self, model, *, head: bool = False, top: int = 0, dtype: str = "bf16", group: int = 128, copies: int = 1, device: str = "cuda", seed: int = 0):
        H, A, K = (int(model[f]) for f in ("hidden", "heads", "kv_heads"))
        d = H // A
        self.torch_dtype, self.dtype = DTYPES[dtype]
        self.hidden, self.group, self.head, self.top = H, group, head, top
        self.device = device = torch.empty(0, device=device).device    # with its number
        self.gen = torch.Generator(device=device)
        self.gen.manual_seed(seed)
        sizes = dict(head=(int(model["vocab"]), H)) if head else \
            dict(qkv=((A + 2 * K) * d, H), out=(H, A * d), gate=(int(model["intermediate"]), H), up=(int(model["intermediate"]), H), down=(H, int(model["intermediate"])))
        with torch.cuda.device(device):
            self.copies = [{f: self._packed(*size) for f, size in sizes.items()} for _ in range(copies)]
        self.sizes = sizes

    def _packed(self, n_out: int, n_in: int) -> dict:
        values = (n_in ** -0.5 * torch.randn((n_out, n_in), generator=self.gen, device=self.device)).to(self.torch_dtype)
        codes, pairs = binding.weight_row_bytes(self.group, n_in)
        w = dict(codes=torch.empty((n_out, codes), dtype=torch.uint8, device=self.device), pairs=torch.empty((n_out, pairs), dtype=torch.uint8, device=self.device))
        w["w"] = binding.make_weights(self.dtype, self.group, n_out, n_in, w["codes"].data_ptr(), w["pairs"].data_ptr())
        binding.ap_weights_pack(w["w"], binding.make_vectors(values.data_ptr(), n_in), torch.cuda.current_stream().cuda_stream)
        return w

    def bytes(self) -> int:
        """Of one copy."""
        return sum(x.numel() for w in self.copies[0].values() for x in (w["codes"], w["pairs"]))

    def plan(self, n_tokens: int) -> dict:
        """Rows, descriptions and workspace of steps of ``n_tokens`` rows: ``x`` goes in, ``y`` comes out (``logits`` and the answers)."""
        if n_tokens < 1:
            raise ValueError(f"a step of {n_tokens} tokens")
        rows = lambda n: torch.zeros((n_tokens, n), dtype=self.torch_dtype, device=self.device)    # noqa: E731
        p = dict(n=n_tokens, at=0, x=torch.randn((n_tokens, self.hidden), generator=self.gen, device=self.device).to(self.torch_dtype))
        w = {f: c["w"] for f, c in self.copies[0].items()}
        with torch.cuda.device(self.device):
            if self.head:
                vocab = self.sizes["head"][0]
                wide = -(-vocab // 8) * 8                  # rows of logits begin at multiples of 16 bytes
                p["y"] = rows(wide)
                p["logits"] = binding.make_logits(self.dtype, n_tokens, vocab, p["y"].data_ptr(), 2 * wide)
                p["tokens"] = torch.zeros(n_tokens, dtype=torch.int32, device=self.device)
                p["logprob"], p["entropy"] = (torch.zeros(n_tokens, device=self.device) for _ in range(2))
                p["top_id"], p["top_logprob"] = (torch.zeros((n_tokens, self.top), dtype=t, device=self.device) for t in (torch.int32, torch.float32))
                need = [binding.ap_linear_workspace(w["head"], n_tokens), binding.ap_logprobs_workspace(p["logits"], self.top)]
            else:
                for f in ("qkv", "gate"):
                    p[f] = rows(self.sizes[f][0])
                p["attended"] = torch.randn((n_tokens, self.sizes["out"][1]), generator=self.gen, device=self.device).to(self.torch_dtype)
                p["mid"], p["y"] = rows(self.hidden), rows(self.hidden)
                need = [binding.ap_linear_workspace(w[f], n_tokens) for f in ("qkv", "out", "down")] + [binding.ap_gated_workspace(w["gate"], w["up"], n_tokens)]
            p["space"] = torch.empty(max(16, *need), dtype=torch.uint8, device=self.device)
        p["rows"] = {f: binding.make_vectors(p[f].data_ptr(), p[f].shape[1]) for f in ("x", "y", "qkv", "gate", "attended", "mid") if f in p}
        return p

    def step(self, p: dict) -> torch.Tensor:
        """A layer: queries, keys and values of ``x`` (to ``qkv``); ``attended`` projected onto ``x``; the feed-forward block onto that.  The
        head: logits of ``x``, and what they say of ``tokens``."""
        w, rows, n, b = {f: c["w"] for f, c in self.copies[p["at"]].items()}, p["rows"], p["n"], binding
        p["at"] = (p["at"] + 1) % len(self.copies)
        with torch.cuda.device(self.device):
            tail = (p["space"].data_ptr(), p["space"].numel(), torch.cuda.current_stream().cuda_stream)
            if self.head:
                b.ap_linear(w["head"], rows["x"], rows["y"], n, None, *tail)
                b.ap_logprobs(p["logits"], p["tokens"].data_ptr(), 1.0, self.top, p["logprob"].data_ptr(), p["entropy"].data_ptr(),
                              p["top_id"].data_ptr(), p["top_logprob"].data_ptr(), *tail)
            else:
                b.ap_linear(w["qkv"], rows["x"], rows["qkv"], n, None, *tail)
                b.ap_linear(w["out"], rows["attended"], rows["mid"], n, rows["x"], *tail)
                b.ap_gated(w["gate"], w["up"], rows["mid"], rows["gate"], n, b.AP_SILU, *tail)
                b.ap_linear(w["down"], rows["gate"], rows["y"], n, rows["mid"], *tail)
        return p["y"]

    def time_us(self, n_tokens: int, repeats: int = 20) -> float:
        """Microseconds of a step among others, as ``ReplicaLayer.time_us``."""
        with torch.cuda.device(self.device):
            p = self.plan(n_tokens)
            return _graph_us(lambda: self.step(p), repeats, self.device)


def weight_times(model, batch: int, prompts, *, dtype: str = "bf16", group: int = 128, top: int = 0, repeats: int = 20):
    """Measured microseconds of a layer's projections and feed-forward block with weights in 4 bits: of a decode step of ``batch``
    sequences, of prefills of ``batch`` prompts of each of ``prompts`` (an array); and of the output head on ``batch`` rows with the log
    probabilities of ``top`` alternatives."""
    def of(head):
        one = ReplicaWeights(model, head=head, top=top, dtype=dtype, group=group)
        copies = max(1, min(repeats, -(-2 * CHIP_CACHE // one.bytes())))         # the chip's caches do not hold them
        return one if copies == 1 else ReplicaWeights(model, head=head, top=top, dtype=dtype, group=group, copies=copies)

    layer = of(False)
    decode, prefill = layer.time_us(batch, repeats), np.array([layer.time_us(batch * int(s), max(2, repeats // 4)) for s in prompts])
    return decode, prefill, of(True).time_us(batch, repeats)


def layer_times(model, batch: int, contexts, prompts, *, dtype: str = "bf16", bits: int = 16, page: int = 16, window: int = 0,
                sinks: int = 0, repeats: int = 20):
    """Measured microseconds of a layer's append and attention: decode steps of ``batch`` sequences at each of ``contexts``,
    prefills of ``batch`` prompts of each of ``prompts``.  ``model`` is a record of ``binding.MODEL_DTYPE``."""
    heads, kv_heads, d = int(model["heads"]), int(model["kv_heads"]), int(model["hidden"]) // int(model["heads"])
    longest = max(*contexts, *prompts)
    size = 2 * batch * (-(-longest // page) * page) * kv_heads * (2 * d if bits == 16 else d // 2 + d // 16)
    layer = ReplicaLayer(batch, longest, heads, kv_heads, d, dtype=dtype, bits=bits, page=page, window=window, sinks=sinks,
                         copies=max(1, min(repeats, -(-4 * CHIP_CACHE // size))))   # as many turns as steps, or half of these bytes between two visits
    return (np.array([layer.time_us(int(c), 1, repeats) for c in contexts]),
            np.array([layer.time_us(int(s), int(s), max(2, repeats // 4)) for s in prompts]))


def _roofline_attention_us(model, gpu, batch, n, c):
    """The roofline's time of one layer's attention: n new tokens a sequence over c tokens."""
    A, K, d, e = float(model["heads"]), float(model["kv_heads"]), float(model["hidden"]) / float(model["heads"]), float(model["weight_bits"]) / 8.0
    flops, nbytes = 4.0 * batch * n * c * A * d, e * (2.0 * batch * n * A * d + 2.0 * batch * c * K * d)
    return flops / np.minimum(flops / nbytes * gpu["hbm_bytes_per_s"], gpu["flops"]) * 1e6


def _op_us(gpu, flops, nbytes):
    return flops / np.minimum(flops / nbytes * gpu["hbm_bytes_per_s"], gpu["flops"]) * 1e6


def _roofline_weights_us(model, gpu, batch, n):
    """The roofline's time of one layer's projections and feed-forward block: n new tokens a sequence."""
    H, I, A, K, e, b = *(float(model[f]) for f in ("hidden", "intermediate", "heads", "kv_heads")), float(model["weight_bits"]) / 8.0, float(batch)
    d = H / A
    wide = (A + 2.0 * K) * d
    return _op_us(gpu, 2.0 * b * n * H * wide, e * (H * wide + b * n * H + b * n * wide)) + \
        _op_us(gpu, 2.0 * b * n * A * d * H, e * (A * d * H + b * n * A * d + b * n * H)) + \
        _op_us(gpu, 6.0 * b * n * H * I, e * (3.0 * H * I + 2.0 * b * n * H + 3.0 * b * n * I))


def _roofline_head_us(model, gpu, batch):
    """The roofline's time of the output head on the last position of each sequence."""
    H, V, e, b = float(model["hidden"]), float(model["vocab"]), float(model["weight_bits"]) / 8.0, float(batch)
    return _op_us(gpu, 2.0 * b * H * V, e * (H * V + b * H + b * V))


def _times(grid, us, longest, what):
    """The lengths and times of a measurement as arrays, or ValueError where they say nothing of lengths up to ``longest``."""
    grid, us = np.asarray(grid, np.float64), np.asarray(us, np.float64)
    if grid.ndim != 1 or len(grid) == 0 or grid.shape != us.shape or not (np.diff(grid) > 0).all() or not grid[0] > 0:
        raise ValueError(f"{what}: lengths have to ascend from above 0, with a time for each")
    if not (np.isfinite(us).all() and (us >= 0).all()):
        raise ValueError(f"{what}: times have to be numbers that are not negative")
    if grid[-1] < longest:
        raise ValueError(f"{what}: measured up to {grid[-1]:g} tokens, and {longest} are needed")
    return grid, us


def _between(length, grid, us):
    """Times at ``length``: between two lengths of the grid the mean of the parabolas through both and either neighbour, which is exact
    where times go as a + b n + c n^2, and never outside of the two's times; the first time below the grid."""
    if len(grid) == 1:
        return np.full(len(length), us[0])
    at = np.clip(length, grid[0], grid[-1])
    i = np.clip(np.searchsorted(grid, at, "right") - 1, 0, len(grid) - 2)
    slope = np.diff(us) / np.diff(grid)
    bend = np.zeros_like(slope)
    if len(grid) > 2:
        of_three = np.diff(slope) / (grid[2:] - grid[:-2])
        bend = np.concatenate([of_three[:1], (of_three[1:] + of_three[:-1]) / 2, of_three[-1:]])
    y = us[i] + (at - grid[i]) * (slope[i] + bend[i] * (at - grid[i + 1]))
    return np.clip(y, np.minimum(us[i], us[i + 1]), np.maximum(us[i], us[i + 1]))


def request_tables(model, gpu, batch: int, prompt_len, out_len, contexts, decode_us, prompts, prefill_us, weights=None):
    """``prefill_us`` and ``tpot_us`` (uint32 [1][R], for ``ap_costtable_set``) of requests on a replica of one GPU: the roofline's
    times with its attention term replaced by the measured ones, interpolated by parabolas between the lengths they were taken at.
    With ``weights``, what ``weight_times`` gives for the same ``prompts``, the terms of projections, feed-forward block and head are
    replaced too.

    Lengths ascend and reach the longest prompt (``prompts``) and the longest context of a decode step (``contexts``), otherwise
    ValueError; what is shorter than the first length takes the first time."""
    prompt, out = np.asarray(prompt_len, np.int64), np.asarray(out_len, np.int64)
    longest = int((prompt + out).max())
    contexts, decode_us = _times(contexts, decode_us, longest - 1, "decode steps")
    prompts, prefill_us = _times(prompts, prefill_us, int(prompt.max()), "prefills")
    group = np.array([(0, 0, 1, batch)], dtype=binding.GROUP_DTYPE)
    pre_ns, prefix_ns, _, _ = binding.ap_roofline_tables(np.array([model], binding.MODEL_DTYPE), np.array([gpu], binding.GPU_DTYPE), group, longest)
    length = np.arange(1, longest + 1, dtype=np.float64)
    layers = float(model["layers"])
    change = lambda grid, us, n: layers * (_between(length, grid, us) - _roofline_attention_us(model, gpu, batch, n, length))   # noqa: E731
    pre = np.asarray(pre_ns, np.float64).reshape(-1)[1:longest + 1] / 1e3 + change(prompts, prefill_us, length)
    step = np.diff(np.asarray(prefix_ns, np.float64).reshape(-1))[1:longest + 1] / 1e3 + change(contexts, decode_us, 1.0)
    if weights is not None:
        w_decode, w_prefill, w_head = weights
        _, w_prefill = _times(prompts, w_prefill, int(prompt.max()), "prefills' weights")
        if not (np.isfinite([w_decode, w_head]).all() and min(w_decode, w_head) >= 0):
            raise ValueError("weights: times have to be numbers that are not negative")
        head = float(w_head) - _roofline_head_us(model, gpu, batch)
        pre = pre + layers * (_between(length, prompts, w_prefill) - _roofline_weights_us(model, gpu, batch, length)) + head
        step = step + layers * (float(w_decode) - _roofline_weights_us(model, gpu, batch, 1.0)) + head
    upto = np.concatenate([[0.0], np.cumsum(step)])          # of contexts 1 .. k
    tpot = (upto[prompt + out - 1] - upto[prompt - 1]) / out
    whole = lambda x: np.maximum(1, np.rint(x)).astype(np.uint32)[None]   # noqa: E731
    return whole(pre[prompt - 1]), whole(tpot)
