"""Log probabilities, entropy and alternatives of rows of logits, against plain sums in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import linear as orc
from paper_2604_07144_amd import binding as b
from tests.linear_harness import stream_of

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, b.AP_BF16), "fp16": (torch.float16, b.AP_FP16), "fp32": (torch.float32, b.AP_FP32)}


def _run(x, tokens, scale=1.0, top=0, dtype="bf16", stream=None, want=("logprob", "entropy")):
    """x [rows][vocab] with unit stride in a row; outputs as arrays, with a place before and behind that has to stay."""
    n, vocab = x.shape
    d = b.make_logits(TYPES[dtype][1], n, vocab, x.data_ptr(), x.stride(0) * x.element_size())
    need = b.ap_logprobs_workspace(d, top)
    space = torch.full((max(16, need),), 0xA5, dtype=torch.uint8, device="cuda")
    out = {f: torch.full((n + 2,), 77.0, device="cuda") for f in ("logprob", "entropy")}
    ids = torch.full((n * top + 2,), 77, dtype=torch.int32, device="cuda")
    tops = torch.full((n * top + 2,), 77.0, device="cuda")
    t = torch.as_tensor(tokens, dtype=torch.int32).cuda()
    ptr = lambda f: out[f][1:].data_ptr() if f in want else 0  # noqa: E731
    b.ap_logprobs(d, t.data_ptr() if "logprob" in want else 0, scale, top, ptr("logprob"), ptr("entropy"), ids[1:].data_ptr() if top else 0,
                  tops[1:].data_ptr() if top else 0, space.data_ptr() if need else 0, need, stream_of(stream))
    torch.cuda.synchronize()
    for y in (*out.values(), ids, tops):
        assert y[0] == 77 and y[-1] == 77
    return {**{f: y[1:-1].double().cpu().numpy() for f, y in out.items()}, "ids": ids[1:-1].view(n, top).cpu().numpy(),
            "tops": tops[1:-1].view(n, top).double().cpu().numpy()}


def _check(got, x, tokens, scale, top, rows=None):
    """Terms of a sum are off by 2^-22 and by 2^-23 for each unit of their exponent; additions in order by at most 2^-24 each, of which a
    lane has one for 2048 entries and as many again within and across lanes.  The entropy has the sums twice, once times the exponent."""
    xx, vocab = x.double().cpu().numpy(), x.shape[1]
    for r in range(len(xx)) if rows is None else rows:
        log, entropy, ids, tops, spread = orc.logprobs(xx[r], int(tokens[r]), scale, top)
        each = 2.0 ** -22 + (vocab / 2048 + 40) * 2.0 ** -24
        tol = each + 2.0 ** -22 * spread
        assert np.array_equal(got["ids"][r], ids), r
        for g, w in [(got["logprob"][r], log), *zip(got["tops"][r], tops)]:
            assert (g == w) or abs(g - w) <= tol + 2.0 ** -22 * abs(w), (r, g, w)
        assert abs(got["entropy"][r] - entropy) <= tol * (2 + spread) + 2.0 ** -22 * (abs(entropy) + spread), (r, got["entropy"][r], entropy)


def _logits(n, vocab, dtype, seed=0, apart=0, spread=3.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = spread * torch.randn((n, vocab + apart), generator=gen, device="cuda")
    return x.to(TYPES[dtype][0])[:, :vocab]


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 64, 65, 511, 1000, 4096, 8191, 32001, 128256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,top,apart", [(1, 5, 0), (5, 64, 3), (3, 1, 1)])
def test_sizes(vocab, dtype, n, top, apart):
    x = _logits(n, vocab, dtype, vocab, apart)
    tokens = np.random.default_rng(vocab).integers(0, vocab, n)
    _check(_run(x, tokens, 1.0, top, dtype), x, tokens, 1.0, top)


@pytest.mark.parametrize("n", [1, 31, 130, 700])
@pytest.mark.parametrize("dtype,scale", [("bf16", 0.7), ("fp32", 2.5)])
def test_numbers_of_rows(n, dtype, scale):
    x = _logits(n, 20011, dtype, n, 2)
    tokens = np.random.default_rng(n).integers(-1, 20011, n)
    _check(_run(x, tokens, scale, 20, dtype), x, tokens, scale, 20, range(0, n, max(1, n // 40)))


@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_at_any_address(offset, dtype):
    """Rows that begin anywhere, with larger values right before and behind them."""
    flat = torch.full((4 * 1003 + 64,), 99.0, dtype=TYPES[dtype][0], device="cuda")
    x = flat[offset:offset + 4 * 1003].view(4, 1003)[:, 1:1001]
    x.copy_(_logits(4, 1000, dtype, offset))
    _check(_run(x, [0, 999, 5, -1], 1.0, 10, dtype), x, [0, 999, 5, -1], 1.0, 10)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [300, 30000])
def test_equal_logits_go_by_the_token(dtype, vocab):
    rng = np.random.default_rng(5)
    rows = [np.zeros(vocab), np.full(vocab, -3.0), rng.integers(0, 3, vocab).astype(float), np.where(rng.random(vocab) < 0.5, 0.0, -0.0),
            np.arange(vocab) // 7 % 100 / 4.0, np.minimum(np.arange(vocab), 200) / 8.0, np.maximum(-np.arange(vocab), -200) / 8.0]
    x = torch.from_numpy(np.array(rows)).to(TYPES[dtype][0]).cuda()
    tokens = rng.integers(0, vocab, len(rows))
    _check(_run(x, tokens, 1.0, 64, dtype), x, tokens, 1.0, 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rising", [True, False])
def test_ordered_rows(dtype, rising):
    """Every entry is the largest yet, or none after the first: the reference is raised all the time."""
    vocab = 40000
    x = torch.linspace(-200.0, 200.0, vocab, device="cuda").to(TYPES[dtype][0])
    x = (x if rising else x.flip(0)).repeat(2, 1).contiguous()
    _check(_run(x, [0, vocab - 1], 1.0, 33, dtype), x, [0, vocab - 1], 1.0, 33)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [50, 20000])
def test_tokens_that_are_ruled_out(dtype, vocab):
    """Some, all but a few, all but one, all; and by the type's lowest value instead."""
    x = _logits(7, vocab, dtype, 3).contiguous()
    x[0, ::3] = -np.inf
    keep = x[1, 17:23].clone()
    x[1] = -np.inf
    x[1, 17:23] = keep
    x[2] = -np.inf
    x[2, vocab - 1] = -5.0
    x[3] = -np.inf
    least = torch.finfo(x.dtype).min
    x[4, 1:] = least
    x[5] = least
    x[6] = torch.finfo(x.dtype).max
    tokens = [0, 0, vocab - 1, 3, 0, 7, 2]
    got = _run(x, tokens, 1.0, 8, dtype)
    assert got["logprob"][0] == got["logprob"][1] == got["logprob"][3] == -np.inf and got["entropy"][3] == 0.0
    assert (got["ids"][3] == -1).all() and (got["tops"][3] == -np.inf).all()
    assert got["logprob"][2] == 0.0 and got["ids"][2].tolist() == [vocab - 1] + [-1] * 7
    _check(got, x, tokens, 1.0, 8, (0, 1, 2))
    assert got["logprob"][4] == 0.0 and got["ids"][4, 0] == 0 and got["ids"][4, 1] == 1
    for r in (5, 6):
        assert abs(got["logprob"][r] + np.log(vocab)) < 1e-5 and abs(got["entropy"][r] - np.log(vocab)) < 1e-5 and got["ids"][r].tolist() == list(range(8))


@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
@pytest.mark.parametrize("vocab", [40, 20000])
def test_what_is_not_a_number(odd, vocab):
    x = _logits(4, vocab, "bf16", 4).contiguous()
    clean = _run(x, [1, 2, 3, -1], 1.0, 4)
    x[1, vocab // 2], x[3, 0] = odd, odd
    got = _run(x, [1, 2, 3, -1], 1.0, 4)
    for r in (0, 2):
        for f in got:
            assert np.array_equal(got[f][r], clean[f][r])
    for r in (1, 3):
        assert np.isnan(got["entropy"][r]) and np.isnan(got["tops"][r]).all()
    assert np.isnan(got["logprob"][1]) and got["logprob"][3] == 0.0
    if odd != odd:
        numbers = torch.where(torch.isnan(x), torch.tensor(-np.inf, device="cuda"), x.float()).double().cpu().numpy()
        for r in (1, 3):
            assert got["ids"][r].tolist() == orc.logprobs(numbers[r], 0, 1.0, 4)[2].tolist()


def test_tokens_outside_of_the_vocabulary_are_none():
    x = _logits(4, 100, "fp32", 6)
    assert (_run(x, [-1, 100, -(1 << 31), (1 << 31) - 1], 1.0, 0, "fp32")["logprob"] == 0.0).all()


@pytest.mark.parametrize("n", [3, 600])
@pytest.mark.parametrize("want", [("logprob",), ("entropy",), ()])
def test_a_part_of_the_answers(n, want):
    x = _logits(n, 20000, "bf16", 8)
    tokens = list(range(n))
    whole, part = _run(x, tokens, 1.0, 3), _run(x, tokens, 1.0, 3, want=want)
    for f in ("logprob", "entropy"):
        assert np.array_equal(part[f], whole[f]) if f in want else (part[f] == 77).all()
    assert np.array_equal(part["ids"], whole["ids"]) and np.array_equal(part["tops"], whole["tops"])


@pytest.mark.parametrize("n", [2, 600])
def test_captured_and_on_another_stream(n):
    x, tokens = _logits(n, 30000, "bf16", 9).contiguous(), torch.arange(n, dtype=torch.int32).cuda()
    d = b.make_logits(b.AP_BF16, n, 30000, x.data_ptr())
    need = b.ap_logprobs_workspace(d, 6)
    space = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    log, ent, tops = (torch.zeros(s, device="cuda") for s in ((n,), (n,), (n, 6)))
    ids = torch.zeros((n, 6), dtype=torch.int32, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        b.ap_logprobs(d, tokens.data_ptr(), 1.0, 6, log.data_ptr(), ent.data_ptr(), ids.data_ptr(), tops.data_ptr(), space.data_ptr(), need, stream_of())
    for i in range(4):
        x.copy_(_logits(n, 30000, "bf16", 20 + i))
        log.zero_(), ids.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = _run(x, tokens.cpu(), 1.0, 6)
        assert np.array_equal(got["ids"], ids.cpu().numpy()) and np.array_equal(got["logprob"], log.double().cpu().numpy())
        assert np.array_equal(got["entropy"], ent.double().cpu().numpy()) and np.array_equal(got["tops"], tops.double().cpu().numpy())


@pytest.mark.parametrize("step", [1e-3, 1e-2])
def test_entropy_and_logprob_against_differences(step):
    """The slope of log p of a token by its own logit is 1 - p, and that of the log sum by the scale the mean logit, which the entropy gives."""
    x = _logits(1, 2000, "fp32", 11).contiguous()
    t = 5
    up, down, here = x.clone(), x.clone(), _run(x, [t], 1.0, 0, "fp32")
    up[0, t] += step
    down[0, t] -= step
    slope = (_run(up, [t], 1.0, 0, "fp32")["logprob"][0] - _run(down, [t], 1.0, 0, "fp32")["logprob"][0]) / (2 * step)
    # second order is at most step^2 / 6; two logs, each off by at most 2^-20
    assert abs(slope - (1 - np.exp(here["logprob"][0]))) <= step ** 2 + 2.0 ** -19 / step
    lz = lambda s: float(x[0, t]) * s - _run(x, [t], s, 0, "fp32")["logprob"][0]   # noqa: E731
    mean = (lz(1 + step) - lz(1 - step)) / (2 * step)
    assert abs(lz(1.0) - mean - here["entropy"][0]) <= 200 * step ** 2 + 2.0 ** -18 / step


def test_far_rows():
    """Rows whose offsets pass 32 bits."""
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GiB of device memory")
    wide = torch.zeros((3, (1 << 29) + 1), dtype=torch.float32, device="cuda")
    x = wide[:, 7:1507]
    x.copy_(_logits(3, 1500, "fp32", 12))
    _check(_run(x, [3, 4, 5], 1.0, 5, "fp32"), x, [3, 4, 5], 1.0, 5)


@pytest.mark.parametrize("dtype,width", [("bf16", 8), ("fp32", 4)])
@pytest.mark.parametrize("lane", [0, 37, 63])
def test_alternatives_that_one_lane_finds(dtype, width, lane):
    """Neighbouring tokens of a span that go up from span to span: one lane writes what the others merge, and new ones follow in the same places."""
    vocab, span = 512 * 40, 512 if dtype == "bf16" else 256
    for n in (2, 600):
        x = torch.full((n, vocab), -9.0, device="cuda")
        at = (torch.arange(vocab // span, device="cuda") * span + lane * width)[:, None] + torch.arange(width, device="cuda")
        x[:, at.flatten()] = torch.arange(at.numel(), device="cuda").float() * 2.0 ** -5
        x = x.to(TYPES[dtype][0]).contiguous()
        tokens = np.full(n, vocab - 1)
        _check(_run(x, tokens, 1.0, 64, dtype), x, tokens, 1.0, 64, (0, n - 1))



@pytest.mark.parametrize("rows", [2, 700])
def test_an_infinity_among_the_largest_numbers(rows):
    """Nothing in 32 bits lies above the largest logits by as much as would raise the reference."""
    x = torch.full((rows, 33000), torch.finfo(torch.float32).max, device="cuda")
    x[1, 32000] = float("inf")
    got = _run(x, [5] * rows, 2.0 ** -120, 2, "fp32")
    assert np.isnan(got["logprob"][1]) and np.isnan(got["entropy"][1]) and np.isnan(got["tops"][1]).all()
    assert np.abs(got["logprob"][0] + np.log(33000)) <= 1e-5



@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("scale", [1.0, 0.7, 2.5])
@pytest.mark.parametrize("vocab", [4097, 65537])
def test_answers_are_rounded_once(dtype, scale, vocab):
    """Tokens far below all others, which are alike: the sum is a power of two to 2^-30, so that log p has one rounding of its own, 2^-24."""
    rng = np.random.default_rng(vocab)
    n = 200
    x = torch.zeros((n, vocab), dtype=TYPES[dtype][0], device="cuda")
    tokens = rng.integers(0, vocab, n)
    x[torch.arange(n), torch.from_numpy(tokens).cuda()] = torch.from_numpy(-30.0 / scale - 60.0 * rng.random(n)).to(x.dtype).cuda()
    got = _run(x, tokens, scale, 2, dtype)
    s = float(np.float32(scale)) * x.double().cpu().numpy()[np.arange(n), tokens]
    want = s - np.log(vocab - 1.0)
    assert (np.abs(got["logprob"] - want) <= np.abs(want) * (2.0 ** -24 + 2.0 ** -30)).all()


@pytest.mark.parametrize("vocab", [2, 3, 7, 100, 1000, 4099, 30011, 128256])
@pytest.mark.parametrize("n", [2, 600])
def test_alike_logits(vocab, n):
    """The sum is the number of tokens, and everything else one rounding."""
    x = torch.full((n, vocab), 3.25, dtype=torch.bfloat16, device="cuda")
    got, want = _run(x, np.arange(n) % vocab, 0.7, 1), np.log(float(vocab))
    for f, y in (("logprob", -want), ("entropy", want), ("tops", -want)):
        assert (np.abs(got[f] - y) <= want * (2.0 ** -24 + 2.0 ** -50)).all(), f



@pytest.mark.parametrize("vocab", [50, 20000])
def test_logits_whose_difference_passes_32_bits(vocab):
    """2^-120 is the least that log2(e) times the scale may be: from there on a difference that passes 32 bits is of a token without
    probability, whose logarithm is a number all the same."""
    x = torch.full((3, vocab), -3e38, device="cuda")
    x[:, vocab - 2] = 3e38
    for scale in (0.25, 1e-30, 2.0 ** -120):
        got = _run(x, [0, vocab - 2, vocab - 1], scale, 3, "fp32")
        far = (float(x[0, 0]) - float(x[0, vocab - 2])) * float(np.float32(scale))
        assert np.abs(got["logprob"] - [far, 0.0, far]).max() <= 2.0 ** -24 * abs(far)
        assert (got["ids"] == [vocab - 2, 0, 1]).all() and np.abs(got["tops"] - [0.0, far, far]).max() <= 2.0 ** -24 * abs(far)
        assert (np.abs(got["entropy"]) <= 2.0 ** -100).all()
