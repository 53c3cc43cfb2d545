"""Attention of many rows over a cache in 4 bits: what decoding keeps, magnitudes it is not made for, and pairs that are not numbers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import attention as orc                        # noqa: E402
from tests.attn_harness import Replica, check              # noqa: E402


def _expected(r, q, scale, window=0, sinks=0):
    """The oracle's rows and a bound for keys, values and weights that are rounded to the 11 bits of fp16: half a step, u = 2^-11,
    of each.  A key's rounding moves a score by u of the sum of |q k| scale and a weight by twice that; the result is rounded once."""
    kv, vv, qq, u = r.values("k"), r.values("v"), q.double().cpu().numpy(), 2.0 ** -11
    want, tol = np.zeros((r.T, r.A, r.d)), np.zeros((r.T, r.A, r.d))
    for t, (s, pos) in enumerate(orc.new_tokens(r.first, r.held, r.T)):
        for h in range(r.A):
            k, v, there = r.gathered(s, kv, h // (r.A // r.K), vv)
            o, mean, seen = orc.attention(qq[t, h], k, v, pos, there, scale, window, sinks)
            want[t, h] = o
            if seen:
                live = (np.abs(k) @ np.abs(qq[t, h]) * scale).max()
                moved = ((r.d + 4) * 2.0 ** -24 + u) * live
                tol[t, h] = mean * (2 * u * (1 + u) + 2 * moved * (1 + moved)) + torch.finfo(r.dtype).eps / 2 * np.abs(o) * (1 + 2.0 ** -7) + 1e-30
                tol[t, h] += seen * 2.0 ** -31 * np.abs(v).max()       # weights below what fp16 holds
    return want, tol


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_codes_keep_eleven_bits(dtype, d):
    """Lowest values far from zero, of which a step is a small part: in bf16 neighbouring codes would be the same number."""
    r = Replica([300, 129], [300, 60], K=1, A=4, d=d, dtype=dtype, bits=4)
    for pairs in (r.kp, r.vp):
        step = 0.01 + 0.002 * r.made(*pairs.shape[:-1], d // 64).abs()
        pairs.copy_(torch.stack([step, 3.0 + step], -1).flatten(-2))
    q = (0.3 * r.made(r.T, r.A, r.d)).to(r.dtype)
    check(r.attend(q, 0.1), *_expected(r, q, 0.1))
    q *= 2.0 ** -9
    check(r.attend(q, 51.2), *_expected(r, q, 51.2))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_by, v_by, q_by", [(2.0 ** -20, 1.0, 2.0 ** 20), (1.0, 2.0 ** -40, 1.0), (2.0 ** 20, 2.0 ** 30, 2.0 ** -20), (2.0 ** 60, 1.0, 2.0 ** -60),
                                              (2.0 ** -60, 2.0 ** -100, 2.0 ** 60), (0.0, 0.0, 1.0)])
def test_all_magnitudes(k_by, v_by, q_by, d):
    """A cache whose numbers are far from 1, as a whole and for some of the keys only."""
    r = Replica([200, 333], [100, 333], K=2, A=4, d=d, bits=4)
    r.kp.copy_(r.kp.float() * k_by)
    r.vp.copy_(r.vp.float() * v_by)
    q = (r.made(r.T, r.A, r.d) * q_by).to(r.dtype)
    check(r.attend(q, 0.09), *r.expected(q, 0.09))
    check(r.attend(q, 0.09, 70, 3), *r.expected(q, 0.09, 70, 3))
    r = Replica([200, 333], [100, 333], K=2, A=4, d=d, bits=4, seed=1)
    r.vp[::5] *= v_by
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    check(r.attend(q, 0.09), *r.expected(q, 0.09))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 1e30])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 100])
def test_pairs_that_a_row_does_not_see(new, d, bad):
    """Unseen slots whose pairs are anything, and pairs that only later tokens see."""
    r = Replica([150, 120], [new, new], page=16, K=1, A=4, d=d, bits=4)
    free = torch.from_numpy(np.setdiff1d(np.arange(r.n_pages), np.unique(r.table[r.table >= 0]))).cuda()
    r.kp[free], r.vp[free] = bad, bad
    for s in range(2):                                      # the rest of the last page
        n = int(r.held[s])
        for x in (r.kp, r.vp):
            x[int(r.table[s, (n - 1) // 16]), :, (n - 1) % 16 + 1:] = bad
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    clean, tol = r.expected(q, 0.1)
    check(r.attend(q, 0.1), clean, tol)
    if new > 1:                                             # position n - 2: seen by the last two tokens only
        for x in (r.kp, r.vp):
            x[int(r.table[0, 148 // 16]), :, 148 % 16] = bad
        got = r.attend(q, 0.1)
        check(got[:new - 2], clean[:new - 2], tol[:new - 2])
        check(got[new:], clean[new:], tol[new:])


def test_queries_that_are_not_numbers():
    """A NaN or an infinity in a query row stays in it."""
    r = Replica([150], [150], K=1, A=4, bits=4)
    q = r.made(r.T, r.A, r.d).to(r.dtype)
    clean, tol = r.expected(q, 0.1)
    q[3, 1, 7], q[77, 0, 64] = float("nan"), float("inf")
    got = r.attend(q, 0.1)
    assert torch.isnan(got[3, 1].float()).all()
    rest = torch.ones((r.T, r.A), dtype=torch.bool)
    rest[3, 1] = rest[77, 0] = False
    check(got[rest.cuda()], clean[rest.numpy()], tol[rest.numpy()])


@pytest.mark.parametrize("new", [1, 3, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype, by", [("bf16", 2.0 ** 20), ("bf16", 2.0 ** 100), ("fp16", 64.0)])
def test_steps_that_stand_apart(dtype, by, d, new):
    """Few rows: values of some keys, and of one group of channels of others, with steps far above the rest's."""
    for held in ([300, 1290, 17], [4000, 2100, 700]):
        r = Replica(held, [new] * 3, K=1, A=4, d=d, dtype=dtype, bits=4, page=20)
        r.vp[::7] *= by
        r.vp[1::7, :, 3, :2] *= by
        q = r.made(r.T, r.A, r.d).to(r.dtype)
        check(r.attend(q, 0.09), *r.expected(q, 0.09))
        r = Replica(held, [new] * 3, K=1, A=4, d=d, dtype=dtype, bits=4, page=20, seed=1)
        for s in range(3):                                  # seen by the last token only
            r.vp[int(r.table[s, (held[s] - 1) // 20]), :, (held[s] - 1) % 20] *= by
        check(r.attend(q, 0.09), *r.expected(q, 0.09))


def test_queries_of_zeros_with_a_tiny_scale():
    r = Replica([150], [150], K=1, A=4, bits=4)
    q = torch.zeros((r.T, r.A, r.d), dtype=r.dtype, device="cuda")
    check(r.attend(q, 1e-20), *r.expected(q, 1e-20))
