"""Shared plumbing of the tests of cache and attention: a paged cache with its sequences on the device, the calls on it, and the
oracle's view of the same memory.  (Not a test module.)"""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention as orc
from paper_2604_07144_amd import binding as b

TYPES = {"bf16": (torch.bfloat16, b.AP_BF16), "fp16": (torch.float16, b.AP_FP16)}


def half_step(dtype):
    """A rounding to the type is off by at most this, relative to the value."""
    return torch.finfo(dtype).eps / 2


class Replica:
    """A cache of ``n_pages`` pages and sequences that hold ``held`` tokens, of which the last ``new`` are new."""

    def __init__(self, held, new, *, K=2, A=4, d=128, page=16, dtype="bf16", bits=16, seed=0, spare=3, slot_major=False, max_kv=None, wide=0):
        self.rng = np.random.default_rng(seed)
        self.dtype, self.code = TYPES[dtype]
        self.K, self.A, self.d, self.page, self.bits = K, A, d, page, bits
        self.held, self.new = np.asarray(held, np.int64), np.asarray(new, np.int64)
        self.S, self.T = len(held), int(self.new.sum())
        pages = -(-np.maximum(self.held, 0) // page)
        self.n_pages, self.width = int(pages.sum()) + spare, max(1, int(pages.max()) + wide)
        order = self.rng.permutation(self.n_pages)
        self.table = np.full((self.S, self.width), -1, np.int32)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.first = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.max_kv = max(1, int(self.held.max())) if max_kv is None else max_kv
        made = lambda *shape: torch.from_numpy(self.rng.standard_normal(shape, dtype=np.float32)).cuda()   # noqa: E731
        self.made = made
        # [page][head][slot], or in memory [page][slot][head]
        lay = lambda n, t: (t(self.n_pages, page, K, n).transpose(1, 2) if slot_major else t(self.n_pages, K, page, n))   # noqa: E731
        if bits == 16:
            self.k, self.v = (lay(d, made).to(self.dtype) for _ in range(2))
            self.kp = self.vp = None
        else:
            byte = lambda *shape: torch.from_numpy(self.rng.integers(0, 256, shape, dtype=np.uint8)).cuda()   # noqa: E731
            self.k, self.v = lay(d // 2, byte), lay(d // 2, byte)
            pair = lambda *shape: torch.stack([x := 0.15 + 0.05 * made(*shape[:-1], shape[-1] // 2).abs(), -7.5 * x], -1).flatten(-2).to(self.dtype)   # noqa: E731
            self.kp, self.vp = lay(d // 32, pair), lay(d // 32, pair)

    def describe(self):
        size = self.k.element_size()
        strides = tuple(size * x for x in self.k.stride()[:3])
        pair_strides = tuple(2 * x for x in self.kp.stride()[:3]) if self.bits == 4 else None
        self.d_first, self.d_held, self.d_table = (torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda() for x in (self.first, self.held, self.table))
        cache = b.make_kv_cache(self.code, self.bits, self.n_pages, self.page, self.K, self.d, self.k.data_ptr(), self.v.data_ptr(),
                                self.kp.data_ptr() if self.bits == 4 else 0, self.vp.data_ptr() if self.bits == 4 else 0, strides, pair_strides)
        batch = b.make_seq_batch(self.S, self.T, max(1, int(self.new.max())), self.max_kv, self.d_first.data_ptr(), self.d_held.data_ptr(),
                                 self.d_table.data_ptr(), self.width)
        return cache, batch

    @staticmethod
    def rows(x):
        return b.make_rows(x.data_ptr(), x.shape[1], x.shape[2], x.element_size() * x.stride(0), x.element_size() * x.stride(1))

    def attend(self, q, scale, window=0, sinks=0, out=None, stream=None, space=None):
        cache, batch = self.describe()
        need = b.ap_attention_workspace(cache, batch, self.A, window, sinks)
        space = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda") if space is None else space
        out = torch.full((self.T, self.A, self.d), 7.0, dtype=self.dtype, device="cuda") if out is None else out
        b.ap_attention(cache, batch, self.rows(q), self.rows(out), self.A, scale, window, sinks, space.data_ptr() if need else 0, need,
                       (stream or torch.cuda.current_stream()).cuda_stream)
        torch.cuda.synchronize()
        return out

    # ---- the oracle's view ----
    def values(self, which):
        """The cache as float64 [page][head][slot][channel]."""
        x, pairs = (self.k, self.kp) if which == "k" else (self.v, self.vp)
        if self.bits == 16:
            return x.double().cpu().numpy()
        codes, pr = x.cpu().numpy(), pairs.double().cpu().numpy()
        out = np.empty((*codes.shape[:3], self.d))
        out[..., 0::2], out[..., 1::2] = codes & 15, codes >> 4
        return np.repeat(pr[..., 1::2], 64, -1) + np.repeat(pr[..., 0::2], 64, -1) * out

    def gathered(self, s, kv, head, vv):
        """Keys and values of a sequence and head in order, and which of them are there."""
        n = int(min(max(self.held[s], 0), self.max_kv))
        k, v, there = np.zeros((n, self.d)), np.zeros((n, self.d)), np.zeros(n, bool)
        for p in range(n):
            at = orc.place(self.table[s], p, self.page, self.n_pages, self.max_kv)
            if at is not None:
                k[p], v[p], there[p] = kv[at[0], head, at[1]], vv[at[0], head, at[1]], True
        return k, v, there

    def expected(self, q, scale, window=0, sinks=0):
        """The oracle's rows and how far a kernel's may be from them.

        Weights are rounded to the 16-bit type once (half a step of each, against the mean of |values|), the result once (half a
        step of itself); scores in 32 bits are off by at most (d + 4) 2^-24 of the sum of |q k| scale, and weights by twice that;
        fp16 weights below 2^-14 by at most 2^-25 each, against the largest |value|, with a sum of weights of at least 1.  In 4 bits
        keys and values may be rounded to the 16-bit type before the products: half a step of each once more, which moves a score
        by half a step of the sum of |q k| scale."""
        kv, vv, qq = self.values("k"), self.values("v"), q.double().cpu().numpy()
        u = half_step(self.dtype)
        want, tol = np.zeros((self.T, self.A, self.d)), np.zeros((self.T, self.A, self.d))
        where = orc.new_tokens(self.first, self.held, self.T)
        cached = {}
        for t, (s, pos) in enumerate(where):
            for h in range(self.A):
                head = h // (self.A // self.K)
                if (s, head) not in cached:
                    cached[s, head] = self.gathered(s, kv, head, vv)
                k, v, there = cached[s, head]
                o, mean, seen = orc.attention(qq[t, h], k, v, pos, there, scale, window, sinks)
                want[t, h] = o
                if seen:
                    live = np.where(there[:, None], np.abs(k), 0.0) @ np.abs(qq[t, h]) * scale
                    moved = (self.d + 4) * 2.0 ** -24 * np.nanmax(live) + (u * np.nanmax(live) if self.bits == 4 else 0.0)
                    tol[t, h] = mean * (u * (1 + u) + 2 * moved * (1 + moved) + (u if self.bits == 4 else 0.0)) + u * np.abs(o) * (1 + 2 * u) + 1e-30
                    if self.dtype == torch.float16:
                        tol[t, h] += seen * 2.0 ** -25 * np.abs(np.where(there[:, None], v, 0.0)).max() + 2.0 ** -25
        return want, tol


def check(got, want, tol):
    g = got.double().cpu().numpy()
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(g - want) / np.maximum(tol, 1e-300)):.3g} times the bound, first at {np.argwhere(bad)[0]}"
