"""Attention where the shape of the call chooses the kernels: batches whose sequences could all have many rows, few tokens over
long sequences that are cut into chunks, and calls on either side of a wavefront's number of sequences."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2604_07144_amd import binding as b              # noqa: E402
from tests.attn_harness import Replica, check              # noqa: E402


def _check(r, window=0, sinks=0):
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    check(r.attend(q, r.d ** -0.5, window, sinks), *r.expected(q, r.d ** -0.5, window, sinks))


@pytest.mark.parametrize("bits", [16, 4])
def test_as_many_tokens_as_if_all_sequences_had_many(bits):
    """max_new times the sequences, but dealt out unequally: the rows beyond max_new are left out, the short sequence is served."""
    r = Replica([150, 90], [149, 1], K=1, A=4, bits=bits)
    cache, batch = r.describe()
    batch.max_new = 75
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    want, tol = r.expected(q, 0.1)
    need = b.ap_attention_workspace(cache, batch, r.A)
    space, out = torch.zeros(max(16, need), dtype=torch.uint8, device="cuda"), torch.full_like(q, 7.0)
    b.ap_attention(cache, batch, r.rows(q), r.rows(out), r.A, 0.1, 0, 0, space.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    check(out[:75], want[:75], tol[:75])
    check(out[149:], want[149:], tol[149:])
    assert (out[75:149] == 7).all()
    _check(Replica([150, 90, 60], [60] * 3, K=1, A=4, bits=bits))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("held, new, window, sinks", [([9000], 34, 0, 0), ([6000, 800], 40, 0, 0), ([5000, 4999], 33, 2500, 70)])
def test_chunks_of_a_long_axis(held, new, window, sinks, d, bits):
    _check(Replica(held, [new] * len(held), K=1, A=1, d=d, bits=bits, page=64), window, sinks)


@pytest.mark.parametrize("n", [63, 64, 65, 66])
def test_sequences_around_a_wavefront(n):
    """Every third sequence without new tokens, the last one without any at all."""
    held = np.random.default_rng(n).integers(1, 50, n)
    new = np.where(np.arange(n) % 3 == 1, 0, held)
    held[-1] = new[-1] = 0
    new[n // 2], held[n // 2] = 70, 75
    _check(Replica(held, new, K=1, A=2, page=8, d=64))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("window, sinks", [(0, 0), (50, 3)])
def test_whole_prompts_with_single_tokens_among_them(window, sinks, bits):
    """Prompts down to one token, and one new token of a sequence that is as long as the longest prompt."""
    held, new = [200, 1, 130, 3, 77, 0, 200, 9], [200, 1, 130, 3, 77, 0, 1, 9]
    _check(Replica(held, new, K=2, A=4, bits=bits, page=20), window, sinks)
