"""How near the attention over the paged cache comes to 64 bits where the 16-bit types are tight: bounds for what the kernels say
they round, and nothing beside it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import attention as orc                        # noqa: E402
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
