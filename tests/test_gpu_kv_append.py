"""Appending to the paged cache and reading back (``ap_kv_append``, ``ap_kv_read``) against the oracle in 64 bits: every row where
the table says, nothing else touched, rotation within the roundings of 32 bits and the one to 16, codes of 4 bits exactly."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from oracle import attention as orc                        # noqa: E402
from paper_2604_07144_amd import binding as b              # noqa: E402
from tests.attn_harness import Replica, half_step          # noqa: E402


def _turn(n, rot):
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()


def _append(r, rot, neighbours, with_q, k=None, v=None, q=None, in_place=False, stream=0):
    k = r.made(r.T, r.K, r.d).to(r.dtype) if k is None else k
    v = r.made(r.T, r.K, r.d).to(r.dtype) if v is None else v
    q = (r.made(r.T, r.A, r.d).to(r.dtype) if q is None else q) if with_q else None
    q0 = q.clone() if with_q else None
    q_out = (q if in_place else torch.full_like(q, 7.0)) if with_q else None
    turn = _turn(r.max_kv, rot) if rot else None
    cache, batch = r.describe()
    b.ap_kv_append(cache, batch, r.rows(k), r.rows(v), b.make_rotation(turn.data_ptr(), r.max_kv, rot, neighbours) if rot else None,
                   r.rows(q) if with_q else None, r.rows(q_out) if with_q else None, r.A if with_q else 0, stream)
    torch.cuda.synchronize()
    return k, v, q0, q_out, turn


def _turned32(x, turn, rot, neighbours, dtype):
    """As the kernel rounds: products and their sum in 32 bits, then to the 16-bit type."""
    x = x.float().cpu().numpy()
    out = x.copy()
    i = np.arange(rot // 2)
    a, c = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
    cs, sn = turn[..., 0], turn[..., 1]
    out[..., a], out[..., c] = x[..., a] * cs - x[..., c] * sn, x[..., a] * sn + x[..., c] * cs
    return torch.from_numpy(out).to(dtype)


def _coded(x16):
    """Pairs and codes of rows in the 16-bit type, in 64 bits."""
    x = x16.double().numpy().reshape(*x16.shape[:-1], -1, 64)
    lo, hi = x.min(-1), x.max(-1)
    want = torch.from_numpy((hi - lo) / 15)
    near = want.float().to(x16.dtype)
    step = (near.view(torch.int16) + (near.double() < want).short()).view(x16.dtype).double().numpy()
    code = np.clip(np.rint((x - lo[..., None]) / np.where(step > 0, step, 1)[..., None]), 0, 15)
    return code.reshape(*x16.shape), step, lo


CASES = [
    dict(held=[1], new=[1]), dict(held=[5, 40, 17], new=[1, 1, 1]), dict(held=[33, 0, 64, 7], new=[33, 0, 10, 7], page=20),
    dict(held=[200, 3], new=[150, 3], page=7, K=5, A=15), dict(held=[70] * 70, new=[2] * 70, page=1, K=1, A=3), dict(held=[9, 90], new=[9, 1], slot_major=True),
]


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 64, None])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", CASES)
def test_rows_in_16_bits(case, dtype, d, rot, neighbours):
    r = Replica(**case, d=d, dtype=dtype, seed=3)
    rot = d if rot is None else rot
    kv, vv = r.values("k"), r.values("v")
    k, v, q, q_out, turn = _append(r, rot, neighbours, with_q=True)
    where = orc.new_tokens(r.first, r.held, r.T)
    u, tab = half_step(r.dtype), turn.cpu().numpy() if rot else None
    kk, vn, qq = k.double().cpu().numpy(), v.double().cpu().numpy(), q.double().cpu().numpy()
    want_k, want_v, tol = kv.copy(), vv.copy(), np.zeros_like(kv)
    got_q = q_out.double().cpu().numpy()

    def off(rows, turned):                                  # two products and a sum in 32 bits, each off by 2^-24 of the larger, and half a step
        big = np.sqrt(2) * np.abs(rows).max(-1, keepdims=True)
        return u * np.abs(turned) * (1 + u) + 4 * 2.0 ** -24 * big + (2.0 ** -25 if dtype == "fp16" else 0.0)

    for t, (s, pos) in enumerate(where):
        page, slot = orc.place(r.table[s], pos, r.page, r.n_pages, r.max_kv)
        rows = orc.turned(kk[t], tab[pos], rot, neighbours) if rot else kk[t]
        want_k[page, :, slot], want_v[page, :, slot] = rows, vn[t]
        tol[page, :, slot] = off(kk[t], rows) if rot else 0.0
        tol[page, :, slot, rot:] = 0.0
        wq = orc.turned(qq[t], tab[pos], rot, neighbours) if rot else qq[t]
        assert (np.abs(got_q[t] - wq) <= (off(qq[t], wq) if rot else 0.0)).all(), t
    assert (np.abs(r.values("k") - want_k) <= tol).all()    # also: every other slot as it was
    assert np.array_equal(r.values("v"), want_v)
    out = [torch.full((r.T, r.K, r.d), 7.0, dtype=r.dtype, device="cuda") for _ in range(2)]
    cache, batch = r.describe()
    b.ap_kv_read(cache, batch, r.rows(out[0]), r.rows(out[1]))
    torch.cuda.synchronize()
    assert torch.equal(out[1], v)
    for t, (s, pos) in enumerate(where):
        page, slot = orc.place(r.table[s], pos, r.page, r.n_pages, r.max_kv)
        assert torch.equal(out[0][t], r.k[page, :, slot]), t


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d, rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 96), (128, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", CASES)
def test_rows_in_4_bits(case, dtype, d, rot, neighbours):
    r = Replica(**case, d=d, dtype=dtype, bits=4, seed=4)
    before = [x.clone() for x in (r.k, r.v, r.kp, r.vp)]
    k, v, q, q_out, turn = _append(r, rot, neighbours, with_q=False)
    out = [torch.full((r.T, r.K, r.d), 7.0, dtype=r.dtype, device="cuda") for _ in range(2)]
    cache, batch = r.describe()
    b.ap_kv_read(cache, batch, r.rows(out[0]), r.rows(out[1]))
    torch.cuda.synchronize()
    where = orc.new_tokens(r.first, r.held, r.T)
    touched = np.zeros((r.n_pages, r.page), bool)
    for which, rows, back in (("k", k, out[0]), ("v", v, out[1])):
        x16 = rows.cpu()
        if which == "k" and rot:
            tab = turn.cpu().numpy()[where[:, 1]][:, None]
            x16 = _turned32(rows, tab, rot, neighbours, r.dtype)
        code, step, lo = _coded(x16)
        got_c, got_p = (getattr(r, which).cpu().numpy(), getattr(r, which + "p").double().cpu().numpy())
        value = (np.repeat(lo, 64, -1) + np.repeat(step, 64, -1) * code)
        for t, (s, pos) in enumerate(where):
            page, slot = orc.place(r.table[s], pos, r.page, r.n_pages, r.max_kv)
            touched[page, slot] = True
            c, p = got_c[page, :, slot], got_p[page, :, slot]
            assert np.array_equal(p[..., 0::2], step[t]) and np.array_equal(p[..., 1::2], lo[t]), (which, t)
            assert np.array_equal(c & 15, code[t][..., 0::2]) and np.array_equal(c >> 4, code[t][..., 1::2]), (which, t)
            # what it stands for is within half a step of what was put in, and comes back as such, rounded once
            assert (np.abs(value[t] - x16[t].double().numpy()) <= 0.5 * np.repeat(step[t], 64, -1) * (1 + 1e-12)).all()
        assert torch.equal(back.cpu(), torch.from_numpy(value).float().to(r.dtype))
    for now, then in zip((r.k, r.v, r.kp, r.vp), before):
        keep = torch.from_numpy(~touched)
        assert torch.equal(now.cpu().transpose(1, 2)[keep].view(torch.uint8), then.cpu().transpose(1, 2)[keep].view(torch.uint8))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extreme_rows(dtype, bits):
    """Values alike, the type's largest of both signs, infinities and NaN: the group that holds one is NaN, the others are as ever."""
    r = Replica([6], [6], dtype=dtype, bits=bits, K=1, A=1)
    big = float(torch.finfo(r.dtype).max)
    k = r.made(6, 1, 128).to(r.dtype)
    k[0] = 3.0
    k[1, 0, :64] = torch.linspace(-1, 1, 64).to(r.dtype) * big
    k[2, 0, 5], k[3, 0, 70], k[4, 0, 1] = float("inf"), float("nan"), float("-inf")
    k[5] = 0.0
    _append(r, 0, False, with_q=False, k=k, v=k)
    out = [torch.zeros((6, 1, 128), dtype=r.dtype, device="cuda") for _ in range(2)]
    cache, batch = r.describe()
    b.ap_kv_read(cache, batch, r.rows(out[0]), r.rows(out[1]))
    torch.cuda.synchronize()
    for x in out:
        if bits == 16:
            assert torch.equal(x.view(torch.int16), k.view(torch.int16))
            continue
        assert torch.equal(x[0], k[0]) and torch.equal(x[5], k[5])
        group = k[1, 0, :64].double()
        step = 2 * big / 15 * (1 + 2 * half_step(r.dtype))
        assert ((x[1, 0, :64].double() - group).abs() <= step * (0.5 + 1e-6) + half_step(r.dtype) * big).all()
        nan = torch.isnan(x[:, 0]).view(6, 2, 64)
        assert nan.all(-1).tolist() == nan.any(-1).tolist() == [[False, False], [False, False], [True, False], [False, True], [True, False], [False, False]]


@pytest.mark.parametrize("bits", [16, 4])
def test_tokens_that_have_no_place(bits):
    """No page in the table, a page id out of range, a position below zero or from max_kv on: nothing is written for them, their
    queries are turned where the position is one and zeros where not, and they read back as zeros."""
    r = Replica([40, 3, 30, -5], [8, 5, 30, 2], bits=bits, page=8, max_kv=36, K=2, A=4)   # sequence 1: positions -2 .. 2; 0: 32 .. 39
    r.table[2, 1], r.table[2, 2], r.table[2, 3] = -1, r.n_pages, 2 ** 31 - 1
    before = [x.clone() for x in (r.k, r.v)]
    k, v, q, q_out, turn = _append(r, 128, False, with_q=True)
    out = [torch.full((r.T, r.K, r.d), 7.0, dtype=r.dtype, device="cuda") for _ in range(2)]
    cache, batch = r.describe()
    b.ap_kv_read(cache, batch, r.rows(out[0]), r.rows(out[1]))
    torch.cuda.synchronize()
    touched = np.zeros((r.n_pages, r.page), bool)
    for t, (s, pos) in enumerate(orc.new_tokens(r.first, r.held, r.T)):
        at = orc.place(r.table[s], pos, r.page, r.n_pages, r.max_kv)
        inside = 0 <= pos < min(r.max_kv, r.held[s])
        assert bool((q_out[t] != 0).any()) == inside, (t, s, pos)
        if at is None or not inside:
            assert not out[0][t].any() and not out[1][t].any()
        else:
            touched[at] = True
            assert bool(out[1][t].any())
    keep = torch.from_numpy(~touched)
    for now, then in zip((r.k, r.v), before):
        assert torch.equal(now.cpu().transpose(1, 2)[keep], then.cpu().transpose(1, 2)[keep])


def test_strided_rows_in_place_and_another_stream():
    r = Replica([50, 20], [50, 1], K=4, A=8, dtype="fp16")
    fused = r.made(r.T, r.A + 2 * r.K, r.d).to(r.dtype)     # queries, keys and values of a token side by side
    plain = fused.clone()
    q, k, v = fused[:, :8], fused[:, 8:12], fused[:, 12:]
    other = Replica([50, 20], [50, 1], K=4, A=8, dtype="fp16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _append(r, 128, True, with_q=True, k=k, v=v, q=q, in_place=True, stream=side.cuda_stream)
    *_, q_out, _ = _append(other, 128, True, with_q=True, k=plain[:, 8:12].contiguous(), v=plain[:, 12:].contiguous(), q=plain[:, :8].contiguous())
    assert torch.equal(r.k, other.k) and torch.equal(r.v, other.v) and torch.equal(fused[:, :8], q_out)
    assert torch.equal(fused[:, 8:], plain[:, 8:])


def test_slots_beyond_4_gib_of_offset():
    """A page far into a cache of more than 2^32 bytes."""
    K, d, page = 8, 128, 16
    n_pages = (1 << 32) // (K * page * d * 2) + 64
    pool = torch.zeros((n_pages, K, page, d), dtype=torch.bfloat16, device="cuda")
    r = Replica([20], [20], K=K, A=8)
    r.k = r.v = pool
    r.n_pages = n_pages
    r.table[0, :2] = n_pages - 1, 3
    k = r.made(20, K, d).to(r.dtype)
    _append(r, 0, False, with_q=False, k=k, v=k)            # keys and values share the memory here, so they are the same rows
    assert torch.equal(pool[n_pages - 1].transpose(0, 1), k[:16]) and torch.equal(pool[3, :, :4].transpose(0, 1), k[16:])
    out = [torch.zeros((20, K, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache, batch = r.describe()
    b.ap_kv_read(cache, batch, r.rows(out[0]), r.rows(out[1]))
    torch.cuda.synchronize()
    assert torch.equal(out[0][16:], pool[3, :, :4].transpose(0, 1)) and torch.equal(out[0][:16], pool[n_pages - 1].transpose(0, 1))
