"""Shared plumbing of the tests of weights in 4 bits: packed matrices on the device, the calls on them, and what the oracle makes of the
same memory.  (Not a test module.)"""
from __future__ import annotations

import numpy as np
import torch

from oracle import linear as orc
from paper_2604_07144_amd import binding as b

TYPES = {"bf16": (torch.bfloat16, b.AP_BF16), "fp16": (torch.float16, b.AP_FP16)}


def half_step(dtype):
    """A rounding to the type is off by at most this, relative to the value."""
    return torch.finfo(dtype).eps / 2


def stream_of(stream=None):
    return (stream or torch.cuda.current_stream()).cuda_stream


def vectors(x):
    return b.make_vectors(x.data_ptr(), x.shape[-1], x.stride(0) * x.element_size() if x.dim() == 2 else 0)


class Matrix:
    """Weights [n_out][n_in] of random codes and pairs, in rows that may be further apart than they are long."""

    def __init__(self, n_out, n_in, group=128, dtype="bf16", seed=0, apart=0, offset=0.3):
        self.n_out, self.n_in, self.group = n_out, n_in, group
        self.dtype, self.code = TYPES[dtype]
        rng = np.random.default_rng(seed)
        blocks = -(-n_in // 128)
        words = rng.integers(0, 1 << 32, (n_out, blocks * 16 + 4 * apart), dtype=np.uint32)
        step = (0.5 + rng.random((n_out, blocks * 128 // group + apart * 128 // group))) * n_in ** -0.5 / 4
        pairs = np.stack([step, -7.5 * step + offset * step * rng.standard_normal(step.shape)], -1)
        self.words = torch.from_numpy(words.view(np.int32)).cuda()
        self.pairs = torch.from_numpy(pairs).to(self.dtype).cuda()

    def describe(self):
        return b.make_weights(self.code, self.group, self.n_out, self.n_in, self.words.data_ptr(), self.pairs.data_ptr(),
                              4 * self.words.stride(0), 2 * self.pairs.stride(0))

    def values(self):
        return orc.values(self.words.cpu().numpy().view(np.uint32), self.pairs.double().cpu().numpy(), self.group, self.n_in)

    def parts(self):
        """|step (16 + code)| + |lo - 16 step| of every weight: what sums in 32 bits are made of."""
        pairs = np.repeat(self.pairs.double().cpu().numpy(), self.group, 1)[:, :self.n_in]
        return np.abs(self.values() - pairs[..., 1] + 16 * pairs[..., 0]) + np.abs(pairs[..., 1] - 16 * pairs[..., 0])

    def linear(self, x, add=None, y=None, n_tokens=None, stream=None, space=None):
        n_tokens = x.shape[0] if n_tokens is None else n_tokens
        y = torch.full((x.shape[0], self.n_out), 7.0, dtype=self.dtype, device="cuda") if y is None else y
        w = self.describe()
        need = b.ap_linear_workspace(w, n_tokens)
        space = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda") if space is None else space
        b.ap_linear(w, vectors(x), vectors(y), n_tokens, None if add is None else vectors(add), space.data_ptr() if need else 0, need, stream_of(stream))
        return y

    def sums(self, x):
        """Products in 64 bits, and how far sums in 32 bits may be from them.

        The factors are exact.  A path through the sums of a group has at most ``group`` additions, a wavefront's then two for each of its groups,
        and 16 more join the wavefronts (and parts of the inputs): each is off by at most 2^-24 of what is summed, by size."""
        xx = x.double().cpu().numpy()
        steps = self.group + 2 * -(-self.n_in // self.group) + 16
        return xx @ self.values().T, steps * 2.0 ** -24 * (np.abs(xx) @ self.parts().T)


def gated(gate, up, x, act="silu", h=None, stream=None, space=None):
    h = torch.full((x.shape[0], gate.n_out), 7.0, dtype=gate.dtype, device="cuda") if h is None else h
    g, u = gate.describe(), up.describe()
    need = b.ap_gated_workspace(g, u, x.shape[0])
    space = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda") if space is None else space
    b.ap_gated(g, u, vectors(x), vectors(h), x.shape[0], {"silu": b.AP_SILU, "gelu": b.AP_GELU}[act], space.data_ptr() if need else 0, need, stream_of(stream))
    return h


def rows(n, k, dtype, seed=0, apart=0):
    """Rows of activations on the device, ``apart`` values more than they are long from one to the next."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn((max(n, 1), k + apart), generator=gen, device="cuda") + 0.1 * torch.randn(k + apart, generator=gen, device="cuda")
    return x.to(TYPES[dtype][0])[:n, :k]


def check_linear(m, x, got, add=None):
    want, tol = m.sums(x)
    if add is not None:
        more = add.double().cpu().numpy()
        tol = tol + 2.0 ** -24 * (np.abs(want) + np.abs(more))
        want = want + more
    check(got, want, tol, m.dtype)


def check_gated(gate, up, x, got, kind):
    """The activation's slope is at most 1.13 and its second derivative below 1; e^-g by a product and a power of two is off by at most
    (4 + |g|) 2^-23 of itself; tanh by 2^-22."""
    (g, eg), (u, eu) = gate.sums(x), up.sums(x)
    a = orc.act(g, kind)
    ea = 1.13 * eg + eg * eg + (np.abs(a) * (4 + np.abs(g)) * 2.0 ** -23 if kind == "silu" else np.abs(g) * (8 + np.minimum(np.abs(g) ** 3, 8)) * 2.0 ** -23)
    check(got, a * u, ea * np.abs(u) + (np.abs(a) + ea) * eu + 2.0 ** -23 * np.abs(a * u), gate.dtype)


def check(got, want, tol, dtype):
    """One rounding beside what sums in 32 bits may be off; and the whole is off by no more than roundings can be."""
    u, least = half_step(dtype), 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134
    g = got.double().cpu().numpy()
    far, bound = np.abs(g - want), tol * (1 + u) + u * np.abs(want) + least
    bad = ~(far <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(far / bound):.3g} times the bound, first at {np.argwhere(bad)[0]}"
    if want.size >= 256:
        assert np.sqrt(np.mean(far ** 2)) <= u * np.sqrt(np.mean(want ** 2)) + least
