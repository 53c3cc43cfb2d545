"""Attention over the paged cache (``ap_attention``) against the oracle in 64 bits; how far a result may be off is derived in
``Replica.expected``."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2604_07144_amd import binding as b              # noqa: E402
from tests.attn_harness import Replica, check              # noqa: E402


def _check(r, window=0, sinks=0, scale=None):
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    scale = r.d ** -0.5 if scale is None else scale
    got = r.attend(q, scale, window, sinks)
    check(got, *r.expected(q, scale, window, sinks))
    return got


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K, A", [(1, 1), (2, 8), (1, 7), (1, 24), (1, 40)])
def test_one_new_token(K, A, dtype, d, bits):
    _check(Replica([1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300], [1] * 12, K=K, A=A, d=d, dtype=dtype, bits=bits))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("page", [1, 7, 16, 48, 256])
def test_page_sizes(page, bits):
    _check(Replica([1, 100, 257], [1, 1, 1], page=page, bits=bits))
    _check(Replica([150, 90], [150, 40], page=page, bits=bits, seed=1))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 3), (5, 2), (32, 0), (33, 40), (100, 4), (100, 64), (1000, 4), (40, 1000)])
@pytest.mark.parametrize("new", [1, 3, 200])
def test_window_and_sinks(new, window, sinks, bits):
    held = np.array([250, 10, 333, 1])
    _check(Replica(held, np.minimum(held, new), K=1, A=4, bits=bits, seed=window), window, sinks)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K, A", [(2, 2), (1, 4), (1, 7), (1, 70)])
def test_many_new_tokens(K, A, dtype, d, bits):
    """Whole prompts, chunks and single tokens side by side."""
    _check(Replica([129, 64, 200, 1, 70, 0, 300], [129, 1, 77, 1, 2, 0, 33], K=K, A=A, d=d, dtype=dtype, bits=bits, page=20))


@pytest.mark.parametrize("new", [2, 4, 8, 16])
def test_a_few_new_tokens(new):
    _check(Replica([40, 16, 500, 129], [new] * 4, K=1, A=4))


SHARES = [(2, 2, 1), (2, 12, 1), (1, 4, 6), (1, 24, 1)]           # key/value heads, query heads, new tokens: 1, 6 and 24 rows of each head


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K, A, new", SHARES)
def test_long_ragged_sequences_dealt_out_evenly(K, A, new, dtype, d, bits):
    """Sequences that are cut anywhere, some of them longer than what a wavefront takes, one empty."""
    held = np.array([1, 2100, 0, 40, 700, 33, 1290, 5])
    _check(Replica(held, np.minimum(held, new), K=K, A=A, d=d, dtype=dtype, bits=bits, page=20))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("K, A, new", [(4, 4, 1), (4, 8, 3), (4, 28, 3)])
def test_many_short_sequences_uncut(K, A, new, d, bits):
    held = np.random.default_rng(6).integers(0, 150, 66)
    _check(Replica(held, np.minimum(held, new), K=K, A=A, d=d, bits=bits, dtype="fp16" if d == 64 else "bf16"))
    _check(Replica(held, np.minimum(held, new), K=K, A=A, d=d, bits=bits, seed=1), window=30, sinks=2)


@pytest.mark.parametrize("bits", [16, 4])
def test_more_sequences_than_a_launch_takes(bits):
    """Long and short ones beyond the 256 of a launch, beside a prompt."""
    held = np.random.default_rng(7).integers(0, 40, 600)
    held[[3, 300, 599]] = 1500, 1300, 200
    new = np.minimum(held, 1)
    new[599] = 150
    _check(Replica(held, new, K=1, A=4, bits=bits))


def test_long_axis_is_split_and_joined():
    _check(Replica([5000, 1, 900], [1, 1, 1], K=1, A=8))
    _check(Replica([4000], [70], K=1, A=2, page=64))
    _check(Replica([3000], [130], K=1, A=2, bits=4, dtype="fp16"), window=900, sinks=7)


def test_many_sequences():
    rng = np.random.default_rng(5)
    held = rng.integers(0, 60, 300)
    _check(Replica(held, np.minimum(held, rng.integers(0, 3, 300)), K=1, A=2, page=8))
    _check(Replica(held, held, K=1, A=3, page=8, d=64))


def test_large_scores_keep_the_maximum():
    """Scores that grow along the keys, far past what an exponential holds without its maximum, and all of them far below zero."""
    for sign in (1.0, -1.0):
        r = Replica([300, 200], [1, 150], K=1, A=4)
        r.k = (torch.arange(r.n_pages * r.page, device="cuda").view(r.n_pages, 1, r.page, 1) * 0.02 + 0.1 * r.made(*r.k.shape)).to(r.dtype)
        q = (sign * (3.0 + 0.2 * r.made(r.T, r.A, r.d))).to(r.dtype)
        check(r.attend(q, 0.3), *r.expected(q, 0.3))


def test_tokens_that_see_nothing():
    """Positions below zero, sequences whose pages are all gone, a window whose pages are gone: zeros; and no page that nobody sees
    is read."""
    r = Replica([3, 40, 200, 100], [10, 40, 1, 60], page=8, K=1, A=4)
    r.table[1, :] = -1
    r.table[2, 2:23] = r.n_pages + 5                        # all that a window of 20 leaves behind
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    got = r.attend(q, 0.1, 20, 0)
    check(got, *r.expected(q, 0.1, 20, 0))
    assert not got[:7].any() and not got[10:50].any() and got[7:10].any() and got[50].any()
    r.table[3, -3:] = 2 ** 31 - 1
    got = r.attend(q, 0.1, 8, 0)
    check(got, *r.expected(q, 0.1, 8, 0))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new", [1, 3, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_seen_does_not_reach_a_row(new, bad, d):
    """Unseen slots full of NaN or infinities, and a value that only later tokens see."""
    r = Replica([150, 120], [new, new], page=16, K=1, A=4, d=d, spare=3)
    used = np.unique(r.table[r.table >= 0])
    free = np.setdiff1d(np.arange(r.n_pages), used)
    r.k[torch.from_numpy(free).cuda()] = bad
    r.v[torch.from_numpy(free).cuda()] = bad
    for s in range(2):                                      # the rest of the last page
        n = int(r.held[s])
        r.k[int(r.table[s, (n - 1) // 16]), :, (n - 1) % 16 + 1:] = bad
        r.v[int(r.table[s, (n - 1) // 16]), :, (n - 1) % 16 + 1:] = bad
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    check(r.attend(q, 0.1), *r.expected(q, 0.1))
    if new > 1:                                             # position n - 2: seen by the last two tokens only
        clean, tol = r.expected(q, 0.1)
        r.v[int(r.table[0, 148 // 16]), :, 148 % 16, 3:40] = bad
        got = r.attend(q, 0.1)
        check(got[:new - 2], clean[:new - 2], tol[:new - 2])
        check(got[new:], clean[new:], tol[new:])
        rows = got[new - 2:new].double().cpu().numpy()
        assert not np.isfinite(rows[..., 3:40]).any()
        check(got[new - 2:new, :, 40:], clean[new - 2:new, :, 40:], tol[new - 2:new, :, 40:])
        # and one that a window hides from the later ones
        r.v[int(r.table[0, 148 // 16]), :, 148 % 16, 3:40] = 1.0
        p = 150 - new
        r.v[int(r.table[0, p // 16]), :, p % 16] = bad      # seen by the first new token, with a window of 1 by no other
        clean, tol = r.expected(q, 0.1, 1, 0)
        got = r.attend(q, 0.1, 1, 0)
        check(got[1:], clean[1:], tol[1:])
        assert not torch.isfinite(got[0].float()).any()


def test_scores_of_nan_and_infinity():
    """A key that is NaN makes the rows that see it NaN; rows whose scores are all minus infinity are zeros."""
    r = Replica([40, 90], [1, 80], K=1, A=2)
    r.k[int(r.table[0, 1]), 0, 3, 7] = float("nan")
    r.k[int(r.table[1, 2]), 0, 8, 0] = float("nan")         # position 40 of sequence 1, whose first new token is at 10
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    want, tol = r.expected(q, 0.1)
    got = r.attend(q, 0.1)
    assert torch.isnan(got[0].float()).all() and torch.isnan(got[1 + 30:].float()).all()
    check(got[1:31], want[1:31], tol[1:31])
    r = Replica([40, 90], [1, 80], K=1, A=2)
    r.k[:] = float("-inf")
    got = r.attend(torch.ones((r.T, 2, 128), dtype=r.dtype, device="cuda"), 0.1)
    assert not got.any()


@pytest.mark.parametrize("new", [1, 60])
def test_strides_streams_and_a_used_workspace(new):
    """Queries and results inside wider rows, a cache that is laid out slot by slot, another stream, results the same every time."""
    r = Replica([700, 60, 333], [new] * 3, K=2, A=8, slot_major=True, wide=5)
    wide_q, wide_o = r.made(r.T, 3 * r.A, r.d + 64).to(r.dtype), torch.full((r.T, r.A + 2, 2 * r.d), 7.0, dtype=r.dtype, device="cuda")
    q, out = wide_q[:, 1:3 * r.A:3, :r.d], wide_o[:, 2:, r.d:]
    want, tol = r.expected(q, 0.09)
    check(r.attend(q, 0.09, out=out), want, tol)
    assert (wide_o[:, :2] == 7).all() and (wide_o[:, :, :r.d] == 7).all()
    first = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache, batch = r.describe()
    space = torch.zeros(b.ap_attention_workspace(cache, batch, r.A), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        out.fill_(3.0)
        torch.cuda.synchronize()
        r.attend(q, 0.09, out=out, stream=side, space=space)
        assert torch.equal(out, first)


def test_a_captured_step_replays():
    """Append and attention of one step in a graph, replayed with new rows and lengths in the same memory."""
    r = Replica([100, 900, 33], [1, 1, 1], K=2, A=8, max_kv=1000, wide=60)
    cache, batch = r.describe()
    k, v, q = (r.made(3, n, 128).to(r.dtype) for n in (2, 2, 8))
    out = torch.zeros_like(q)
    need = b.ap_attention_workspace(cache, batch, 8)
    space = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    turn = torch.ones((1000, 64, 2), device="cuda") * 0.5 ** 0.5

    def step():
        stream = torch.cuda.current_stream().cuda_stream
        b.ap_kv_append(cache, batch, r.rows(k), r.rows(v), b.make_rotation(turn.data_ptr(), 1000, 128), r.rows(q), r.rows(q), 8, stream)
        b.ap_attention(cache, batch, r.rows(q), r.rows(out), 8, 0.1, 0, 0, space.data_ptr(), need, stream)

    graph = torch.cuda.CUDAGraph()
    start = [x.clone() for x in (r.k, r.v, q)]
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for x, y in zip((r.k, r.v, q), start):
            x.copy_(y)
        q.mul_(1.0 + i)
        r.d_held.copy_(torch.tensor([100 - i, 900 - 2 * i, 33 - i]))
        keep = [x.clone() for x in (r.k, r.v, q)]
        step()
        torch.cuda.synchronize()
        want = out.clone()
        for x, y in zip((r.k, r.v, q), keep):
            x.copy_(y)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(want.any()), i


@pytest.mark.parametrize("bits", [16, 4])
def test_offsets_beyond_32_bits(bits):
    """Pages on either side of 4 GiB, for one token and for many."""
    K, d, page = 8, 128, 64
    row = 2 * d if bits == 16 else d // 2
    n_pages = (1 << 32) // (K * page * row) + 64
    r = Replica([200, 130], [1, 100], K=K, A=8, page=page, bits=bits)
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    want, tol = r.expected(q, 0.1)
    small = dict(k=r.k, v=r.v, kp=r.kp, vp=r.vp)
    for f, x in small.items():
        if x is not None:
            pool = torch.zeros((n_pages, *x.shape[1:]), dtype=x.dtype, device="cuda")
            pool[n_pages - len(x):] = x
            setattr(r, f, pool)
    r.table = np.where(r.table >= 0, r.table + (n_pages - r.n_pages), -1).astype(np.int32)
    r.n_pages = n_pages
    check(r.attend(q, 0.1), want, tol)


def test_many_new_tokens_beyond_max_new_are_left_out():
    r = Replica([60, 40], [30, 1], K=1, A=4)
    cache, batch = r.describe()
    batch.max_new = 10
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    want, tol = r.expected(q, 0.1)
    need = b.ap_attention_workspace(cache, batch, r.A)
    space, out = torch.zeros(max(16, need), dtype=torch.uint8, device="cuda"), torch.full_like(q, 7.0)
    b.ap_attention(cache, batch, r.rows(q), r.rows(out), r.A, 0.1, 0, 0, space.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    check(out[:10], want[:10], tol[:10])
    check(out[30:], want[30:], tol[30:])
    assert (out[10:30] == 7).all()
