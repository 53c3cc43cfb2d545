"""Cost tables with the cache and attention measured on the card.

The roofline prices every operator of a model analytically.  What goes by the lengths in a trace is the cache of keys and
values and the attention over it; this module runs those (``ap_kv_append``, ``ap_attention``) on the present device at a grid of
lengths and puts the measured times in the place of the roofline's attention term, so that ``ap_costtable_set`` can score
candidates with them.  Projections, output head and all-reduce stay the roofline's.
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
            self.step(p)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                for _ in range(repeats):
                    self.step(p)
            other, times = torch.zeros(2 * CHIP_CACHE // 4, dtype=torch.int32, device=self.device), []
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


def request_tables(model, gpu, batch: int, prompt_len, out_len, contexts, decode_us, prompts, prefill_us):
    """``prefill_us`` and ``tpot_us`` (uint32 [1][R], for ``ap_costtable_set``) of requests on a replica of one GPU: the roofline's
    times with its attention term replaced by the measured ones, interpolated by parabolas between the lengths they were taken at.

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
    upto = np.concatenate([[0.0], np.cumsum(step)])          # of contexts 1 .. k
    tpot = (upto[prompt + out - 1] - upto[prompt - 1]) / out
    whole = lambda x: np.maximum(1, np.rint(x)).astype(np.uint32)[None]   # noqa: E731
    return whole(pre[prompt - 1]), whole(tpot)
