"""How near the attention over the paged cache comes to 64 bits where the 16-bit types are tight: bounds for what the kernels say
they round, and nothing beside it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import attention as orc                        # noqa: E402
from paper_2604_07144_amd import binding as b              # noqa: E402
from tests.attn_harness import Replica, check              # noqa: E402


def _rows(r, q, scale, tokens, own_error, window=0, sinks=0):
    """The oracle's rows of some tokens, all heads, and bounds: ``own_error(mean, seen, live, k, v)`` is what a kernel's roundings of
    keys, values and weights may do to a row; its final rounding is half a step of itself."""
    kv, vv, qq = r.values("k"), r.values("v"), q.double().cpu().numpy()
    where, cached = orc.new_tokens(r.first, r.held, r.T), {}
    want, tol = np.zeros((len(tokens), r.A, r.d)), np.zeros((len(tokens), r.A, r.d))
    for i, t in enumerate(tokens):
        s, pos = where[t]
        for h in range(r.A):
            head = h // (r.A // r.K)
            if (s, head) not in cached:
                cached[s, head] = r.gathered(s, kv, head, vv)
            k, v, there = cached[s, head]
            o, mean, seen = orc.attention(qq[t, h], k, v, pos, there, scale, window, sinks)
            live = (np.abs(k) @ np.abs(qq[t, h])).max() * scale
            want[i, h] = o
            tol[i, h] = own_error(mean, seen, live, k, v) + torch.finfo(r.dtype).eps / 2 * np.abs(o) * (1 + 2.0 ** -7) + 1e-30
    return want, tol


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("K, A, new", [(1, 1, 1), (2, 8, 1), (1, 4, 6), (1, 4, 40)])
@pytest.mark.parametrize("held", [300, 3000, 32768])
def test_many_small_weights_in_fp16(held, K, A, new, d):
    """One key with the maximum and a value of zero, and behind it keys whose weights are 2^-24 to 2^-27 of it: their sum is the row.

    Weights are rounded once (half a step, 2^-11), and what the type's range takes of one is at most half of 2^-24 with the maximum's
    at 2^7, so 2^-32 of a value; scores in 32 bits move a weight by 2 (d + 4) 2^-24 of the sum of |q k| scale."""
    r = Replica([held], [new], K=K, A=A, d=d, dtype="fp16", page=64)
    r.k.zero_()
    p = torch.from_numpy(r.table[0, :-(-held // 64)].astype(np.int64)).cuda()
    r.k[p, :, :, 0] = (24.0 + 3.0 * torch.rand(r.k.shape[:3], device="cuda")).to(r.dtype)[p]
    r.k[p[0], :, 0, 0] = 0.0
    r.v[p] = r.v[p].abs() + 0.5
    r.v[p[0], :, 0] = 0.0
    q = torch.zeros((r.T, r.A, d), dtype=r.dtype, device="cuda")
    q[..., 0] = -1.0
    scale, u = float(np.log(2.0)), 2.0 ** -11

    def own(mean, seen, live, k, v):
        moved = 2 * (d + 4) * 2.0 ** -24 * live
        return mean * (u * (1 + u) + moved * (1 + moved)) + seen * 2.0 ** -32 * np.abs(v).max() + 2.0 ** -25

    tokens = [0, new // 2, new - 1]
    want, tol = _rows(r, q, scale, tokens, own)
    check(r.attend(q, scale)[tokens], want, tol)


def _code_error(r, q, scale):
    """Bounds for few rows over 4 bits, where codes are multiplied as they are and nothing but each weight, times its key's step, is rounded
    to 16 bits.

    A weight meets what its code is off the middle one, at most 8 steps, so its rounding is worth half a step of the type of that.  In
    32 bits a score is put together of step * (codes . q) and lo * (sum of q), so what it is off by goes by the sum of |q| times
    |lo| + 15 |step|, and a weight by twice that; the sums of values by what they have added up, 15 steps and |lo|.  fp16 holds weights
    times their steps, 2^10 at the largest step, to half of 2^-24."""
    pairs = {f: x.double().cpu().numpy() for f, x in (("k", r.kp), ("v", r.vp))}
    held = np.isin(np.arange(r.n_pages), r.table[r.table >= 0])
    step, lo = np.abs(pairs["v"][held][..., 0::2]).max(), np.abs(pairs["v"][held][..., 1::2]).max()
    key = (np.abs(pairs["k"][held][..., 1::2]) + 15 * np.abs(pairs["k"][held][..., 0::2])).max()
    u = torch.finfo(r.dtype).eps / 2
    sums = np.abs(q.double().cpu().numpy()).sum(-1).max() * scale * key

    def own(mean, seen, live, k, v):
        moved = 2 * (r.d + 8) * 2.0 ** -24 * sums
        lost = seen * 2.0 ** -31 * step if r.dtype == torch.float16 else 0.0
        return 8 * step * u + mean * moved * (1 + moved) + (seen / 16 + 40) * 2.0 ** -24 * (15 * step + lo) + lost + (2.0 ** -25 if r.dtype == torch.float16 else 0.0)

    return own


def _code_rows(r, q, scale, tokens, window=0, sinks=0):
    return _rows(r, q, scale, tokens, _code_error(r, q, scale), window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("K, A, new", [(1, 4, 1), (2, 2, 1), (1, 24, 1), (1, 4, 6)])
@pytest.mark.parametrize("dtype, k_by, q_by, by", [
    ("bf16", 1, 1, 1), ("fp16", 1, 1, 1), ("fp16", 2.0 ** -6, 2.0 ** 10, 2.0 ** -4), ("fp16", 8, 2.0 ** -8, 32), ("fp16", 1, 2.0 ** -9, 2.0 ** 9),
    ("bf16", 2.0 ** -100, 2.0 ** 60, 2.0 ** 40), ("bf16", 2.0 ** -118, 2.0 ** 118, 1), ("bf16", 2.0 ** -118, 1, 2.0 ** 118), ("bf16", 2.0 ** 110, 2.0 ** -60, 2.0 ** -50),
    ("bf16", 2.0 ** 100, 2.0 ** -100, 1), ("bf16", 1, 2.0 ** -120, 2.0 ** 120), ("bf16", 1, 2.0 ** 120, 2.0 ** -120), ("bf16", 2.0 ** -60, 2.0 ** -60, 2.0 ** 120)])
def test_few_rows_over_4_bits_round_weights_only(dtype, k_by, q_by, by, K, A, new, d):
    """Scores of ordinary size made of keys, queries and scales of any."""
    for held in ([300, 77, 32], [4000, 2100, 700]):
        r = Replica(held, [new] * 3, K=K, A=A, d=d, dtype=dtype, bits=4, page=20)
        r.kp.copy_(r.kp.float() * k_by)
        q = (r.made(r.T, r.A, r.d) * q_by).to(r.dtype)
        tokens, scale = [0, new, 3 * new - 1], d ** -0.5 * by
        check(r.attend(q, scale)[tokens], *_code_rows(r, q, scale, tokens))
        check(r.attend(q, scale, 70, 3)[tokens], *_code_rows(r, q, scale, tokens, 70, 3))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new", [1, 3, 60])
def test_scales_that_leave_no_score(new, bits):
    """A scale below the smallest normal number: every key that is seen has the same weight."""
    r = Replica([200, 333], [new, new], K=1, A=4, bits=bits)
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    check(r.attend(q, 1e-42, 90, 2), *r.expected(q, 1e-42, 90, 2))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K, A, held, new", [(1, 4, 40, 1), (1, 4, 300, 1), (4, 4, 4000, 1), (1, 4, 700, 6), (1, 24, 700, 1), (1, 4, 300, 100), (1, 4, 5000, 40)])
def test_equal_values_come_back_as_they_are(K, A, held, new, dtype, d, bits):
    """All values of a channel alike, under weights that all round the same way: a row is a mean of one value, which is that value.

    The value lies just below a power of two, where half a step is the smallest part of it; weights in 16 bits are taken off it by nearly
    half a step of theirs at the bottom of their step, twice that part.  32 bits leave 2^-14 of half a step beside that."""
    r = Replica([held] * 3, [new] * 3, K=K, A=A, d=d, dtype=dtype, bits=bits, page=20)
    u = torch.finfo(r.dtype).eps / 2
    value = 2.0 - 2 * u
    if bits == 16:
        r.k.zero_()
        r.k[..., 0] = -1.0
        for s in range(3):
            r.k[int(r.table[s, 0]), :, 0, 0] = 0.0          # the first key has the maximum
        r.v[:] = value
    else:                                                   # steps of zero: lo alone
        r.kp.zero_()
        r.kp[..., 1] = -1.0
        for s in range(3):
            r.kp[int(r.table[s, 0]), :, 0, 1] = 0.0
        r.vp.zero_()
        r.vp[..., 1::2] = value
    q = torch.zeros((r.T, A, d), dtype=r.dtype, device="cuda")
    q[..., 0] = 1.0
    scale = -float(np.log(0.5 * (1 + u * (1 - 2.0 ** -3))))
    got = r.attend(q, scale)
    assert (got.double() == value).all(), (got.double().min().item(), got.double().max().item(), value)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("held, new", [(150, 60), (300, 300), (3000, 130)])
@pytest.mark.parametrize("size", [2.0 ** -6, 2.0 ** -7, 2.0 ** -9])
def test_small_groups_keep_eleven_bits(size, held, new, d):
    """Many rows over 4 bits whose groups are small as a whole: neighbouring codes, which bf16 would round apart or together, still
    give their own scores, and values of the same size.

    Keys and values are rounded to 11 bits (u = 2^-11 of each) and lose at most 17 * 2^-25 by the range of fp16; a key's error moves a
    score by that much of the sum of |q| scale, and a weight by twice that."""
    r = Replica([held], [new], K=1, A=4, d=d, bits=4)
    odd = torch.from_numpy(r.rng.integers(0, 2, (r.n_pages, 1, r.page, 1), dtype=np.uint8)).cuda()
    r.k[:] = 0x11 + 0x22 * odd                              # codes 1 and 3, half-way between numbers of bf16: to 0 and to 4
    r.v[:] = 0xFF * odd
    r.kp[..., 0::2], r.kp[..., 1::2] = size / 256, size
    r.vp[..., 0::2], r.vp[..., 1::2] = size / 8, -size * 15 / 16
    q = torch.ones((r.T, r.A, d), dtype=r.dtype, device="cuda")
    scale, u, lost = 64 / (d * size), 2.0 ** -11, 17 * 2.0 ** -25

    def own(mean, seen, live, k, v):
        moved = ((d + 4) * 2.0 ** -24 + u) * live + scale * d * lost
        return mean * (2 * u * (1 + u) + 2 * moved * (1 + moved)) + lost + seen * 2.0 ** -31 * size

    tokens = [0, new // 3, new - 1]
    check(r.attend(q, scale)[tokens], *_rows(r, q, scale, tokens, own))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d, A, new, longest", [(64, 16, 1, 32640), (64, 16, 1, 32641), (64, 40, 3, 32641), (128, 160, 1, 16256), (128, 160, 1, 16257), (128, 40, 5, 16257)])
def test_lines_of_4_bits_on_either_side_of_twice_the_wavefronts(d, A, new, longest, dtype):
    """The lengths from which the kernel of few rows over 4 bits puts twice as many wavefronts on a SIMD (64 channels up to 16 rows, 128
    channels from 17 to 32), the last ones below, and what stands in the workspace then."""
    K, held = 8, np.array([longest, 5, longest // 2, 3000])
    r = Replica(held, np.minimum(held, new), K=K, A=A, d=d, dtype=dtype, bits=4, page=64, wide=2)
    cache, batch = r.describe()
    above, below = (b.ap_attention_workspace(cache, b.make_seq_batch(4, r.T, new, n, 64, 64, 64, r.width), A) for n in (longest + 64, longest - 64))
    need = b.ap_attention_workspace(cache, batch, A)
    assert above > 1.9 * below and need == (above if longest % 32 else below)
    q = (0.5 * r.made(r.T, A, d)).to(r.dtype)
    got, scale = r.attend(q, d ** -0.5).double().cpu().numpy(), d ** -0.5
    own, where, qq = _code_error(r, q, scale), orc.new_tokens(r.first, r.held, r.T), q.double().cpu().numpy()
    for s, head in ((0, 0), (0, K - 1), (1, 3), (2, 5), (3, K - 1)):
        j = torch.arange(int(held[s]), device="cuda")
        page, slot = torch.from_numpy(r.table[s].astype(np.int64)).cuda()[j // 64], j % 64
        rows = []
        for codes, pairs in ((r.k, r.kp), (r.v, r.vp)):
            c, two = codes[page, head, slot].cpu().numpy(), pairs[page, head, slot].double().cpu().numpy()
            rows.append(np.repeat(two[:, 1::2], 64, 1) + np.repeat(two[:, 0::2], 64, 1) * np.stack([c & 15, c >> 4], -1).reshape(len(c), d))
        for t in (int(r.first[s]), int(r.first[s + 1]) - 1):
            for h in (head * (A // K), (head + 1) * (A // K) - 1):
                o, mean, seen = orc.attention(qq[t, h], *rows, where[t, 1], np.ones(len(j), bool), scale, 0, 0)
                tol = own(mean, seen, None, *rows) + torch.finfo(r.dtype).eps / 2 * np.abs(o) * (1 + 2.0 ** -7) + 1e-30
                assert (np.abs(got[t, h] - o) <= tol).all(), (s, t, h, np.max(np.abs(got[t, h] - o) / tol))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("held", [200, 3000])
def test_queries_of_few_rows_that_are_not_numbers(held, dtype, bits):
    """A NaN or an infinity in a query row stays in it, beside rows of any size and of zeros."""
    r = Replica([held] * 3, [2] * 3, K=1, A=4, d=128, dtype=dtype, bits=bits)
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    q[1, 2] = 0.0
    q[4, 1] *= 2.0 ** -12
    clean, tol = r.expected(q, 0.1)
    q[0, 1, 7], q[3, 0, 64], q[5, 3, 127] = float("nan"), float("inf"), float("-inf")
    got = r.attend(q, 0.1)
    assert torch.isnan(got[0, 1].float()).all()
    rest = np.ones((r.T, r.A), dtype=bool)
    rest[0, 1] = rest[3, 0] = rest[5, 3] = False
    check(got[torch.from_numpy(rest).cuda()], clean[rest], tol[rest])
