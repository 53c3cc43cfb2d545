"""Packing weights in 4 bits and reading them back: bit by bit what the rule gives."""
import numpy as np
import pytest
import torch

from oracle import linear as orc
from paper_2604_07144_amd import binding as b
from tests.linear_harness import TYPES, stream_of, vectors

pytestmark = pytest.mark.gpu


def _up(dtype):
    """A float64 of 32 bits rounded up to the type."""
    def up(x):
        y = torch.tensor(x, dtype=torch.float64).float().to(dtype)
        if float(y) < x:
            y = (y.view(torch.int16) + 1).view(dtype)
        return float(y)
    return up


def _pack(x, group, dtype, apart=0):
    """Packs rows; returns (words, pairs) as they lie on the device and the description."""
    n_out, n_in = x.shape
    blocks = -(-n_in // 128)
    words = torch.full((n_out + 1, blocks * 16 + 4 * apart), 0x5A5A5A5A, dtype=torch.int32, device="cuda")
    pairs = torch.full((n_out + 1, blocks * 128 // group + apart * 128 // group, 2), 9.0, dtype=TYPES[dtype][0], device="cuda")
    w = b.make_weights(TYPES[dtype][1], group, n_out, n_in, words.data_ptr(), pairs.data_ptr(), 4 * words.stride(0), 2 * pairs.stride(0))
    b.ap_weights_pack(w, vectors(x), stream_of())
    torch.cuda.synchronize()
    assert (words[n_out] == 0x5A5A5A5A).all() and (pairs[n_out] == 9.0).all()
    assert (words[:, blocks * 16:] == 0x5A5A5A5A).all() and (pairs[:, blocks * 128 // group:] == 9.0).all()
    return words[:n_out, :blocks * 16], pairs[:n_out, :blocks * 128 // group], w, (words, pairs)


def _codes(words, n_in):
    """Codes of all columns of the blocks."""
    w = words.cpu().numpy().view(np.uint32)
    out = np.zeros((w.shape[0], w.shape[1] * 8), np.int64)
    for c in range(out.shape[1]):
        word, bit = orc.place(c)
        out[:, c] = w[:, word] >> np.uint32(bit) & np.uint32(15)
    return out[:, :n_in], out[:, n_in:]


@pytest.mark.parametrize("n_out,n_in,apart", [(1, 8, 0), (3, 24, 1), (5, 128, 0), (17, 136, 1), (70, 376, 0), (9, 1000, 2), (260, 512, 0)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_codes_and_pairs(n_out, n_in, apart, group, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n_out * n_in)
    x = torch.randn((n_out, n_in + 8 * apart), generator=gen, device="cuda").to(TYPES[dtype][0])[:, :n_in]
    words, pairs, w, _keep = _pack(x, group, dtype, apart)
    codes, want = orc.packed(x.double().cpu().numpy(), group, _up(TYPES[dtype][0]))
    got, beyond = _codes(words, n_in)
    assert np.array_equal(pairs.double().cpu().numpy(), want) and np.array_equal(got, codes) and not beyond.any()
    back = torch.full((n_out + 1, n_in + 8), 5.0, dtype=x.dtype, device="cuda")
    b.ap_weights_read(w, b.make_vectors(back.data_ptr(), n_in, 2 * back.stride(0)), stream_of())
    torch.cuda.synchronize()
    stand = torch.from_numpy(orc.values(words.cpu().numpy().view(np.uint32), want, group, n_in)).float().to(x.dtype)
    assert torch.equal(back[:n_out, :n_in].cpu(), stand)
    assert (back[n_out:] == 5.0).all() and (back[:, n_in:] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_on_the_edge(dtype):
    t = TYPES[dtype][0]
    most = torch.finfo(t).max
    x = torch.zeros((8, 256), dtype=t, device="cuda")
    x[1] = 3.25                                                # all alike: a step of zero
    x[2, :128:2], x[2, 1:128:2] = most, -most                  # the widest range there is
    x[3, 5], x[3, 200] = float("nan"), float("inf")            # not numbers: their groups are marked, the others are not
    x[4, 7] = float("-inf")
    x[5] = torch.arange(256, device="cuda").to(t)
    x[6] = -x[5]
    x[7, 3] = torch.finfo(t).tiny
    words, pairs, w, _keep = _pack(x, 64, dtype)
    p, codes = pairs.double().cpu().numpy(), _codes(words, 256)[0]
    assert not codes[:2].any() and (p[1] == [0.0, 3.25]).all()
    odd = np.isnan(p).all(-1)
    assert odd[3].tolist() == [True, False, False, True] and odd[4].tolist() == [True, False, False, False]
    assert np.isfinite(p[~odd]).all()
    back = torch.empty((8, 256), dtype=t, device="cuda")
    b.ap_weights_read(w, vectors(back), stream_of())
    got = back.double().cpu().numpy()
    assert np.isnan(got[3, :64]).all() and np.isnan(got[3, 192:]).all() and (got[3, 64:192] == 0).all()
    assert np.isfinite(got[2]).all() and (np.abs(got[2, :128]) >= 0.93 * most).all()       # a step rounded down loses at most 15 half steps of 1/15th
    # off by at most half a step of the group (which rounding up makes longer by one rounding), and a rounding
    u = torch.finfo(t).eps / 2
    for r in (5, 6):
        assert np.abs(got[r] - x[r].double().cpu().numpy()).max() <= 63 / 15 / 2 * (1 + 2 * u) + u * 255


@pytest.mark.parametrize("group", [32, 128])
def test_many_blocks(group):
    """More blocks than a workgroup takes, and rows that begin anywhere in one."""
    x = torch.randn((301, 1160), device="cuda").bfloat16()
    words, pairs, w, _keep = _pack(x, group, "bf16")
    codes, want = orc.packed(x[::50].double().cpu().numpy(), group, _up(torch.bfloat16))
    assert np.array_equal(_codes(words[::50], 1160)[0], codes) and np.array_equal(pairs[::50].double().cpu().numpy(), want)


def test_captured():
    x = torch.randn((64, 640), device="cuda").half()
    words, pairs, w, keep = _pack(x, 64, "fp16")
    want, back = words.clone(), torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ap_weights_pack(w, vectors(x), stream_of())
        b.ap_weights_read(w, vectors(back), stream_of())
    for _ in range(3):
        keep[0].zero_()
        back.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(words, want) and (back - x).abs().max() < 0.5


@pytest.mark.parametrize("dtype,scale", [("bf16", 1e-30), ("bf16", 1e-4), ("bf16", 1.0), ("bf16", 1e30), ("fp16", 1e-4), ("fp16", 1.0), ("fp16", 1e3)])
def test_values_of_any_size(dtype, scale):
    """Steps from next to nothing to next to overflow, and values that lie in the middle between two codes."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    x = (scale * torch.randn((64, 512), generator=gen, device="cuda")).to(TYPES[dtype][0])
    x[32:] = (scale * (torch.randint(0, 31, (32, 512), generator=gen, device="cuda") / 2.0)).to(x.dtype)
    words, pairs, w, _keep = _pack(x, 64, dtype)
    codes, want = orc.packed(x.double().cpu().numpy(), 64, _up(x.dtype))
    assert np.array_equal(pairs.double().cpu().numpy(), want) and np.array_equal(_codes(words, 512)[0], codes)
