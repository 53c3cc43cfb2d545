"""Products with weights in 4 bits, and the gated half of a feed-forward block, against plain sums in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2604_07144_amd import binding as b
from tests.linear_harness import Matrix, check_gated, check_linear, gated, half_step, rows, stream_of, vectors

pytestmark = pytest.mark.gpu

TOKENS = [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 129, 257, 300, 513]
SIZES = [(1, 8), (7, 24), (16, 128), (17, 120), (33, 136), (100, 1000), (250, 512), (129, 2184), (300, 4096)]


@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("dtype,group", [("bf16", 128), ("fp16", 64), ("bf16", 32)])
def test_numbers_of_tokens(tokens, dtype, group):
    m = Matrix(96 + tokens % 37, 640 + 8 * (tokens % 5), group, dtype, seed=tokens)
    x = rows(tokens, m.n_in, dtype, seed=tokens)
    check_linear(m, x, m.linear(x))


@pytest.mark.parametrize("n_out,n_in", SIZES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens", [1, 9, 40, 150])
def test_sizes(n_out, n_in, group, tokens):
    dtype = "bf16" if (n_out + group) % 3 else "fp16"
    m = Matrix(n_out, n_in, group, dtype, seed=n_out)
    x = rows(tokens, n_in, dtype, seed=n_in)
    check_linear(m, x, m.linear(x))


@pytest.mark.parametrize("tokens", [3, 70, 600])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_outputs_and_inputs(tokens, dtype):
    m = Matrix(1111, 2048 + 64, 64, dtype, seed=tokens)
    x = rows(tokens, m.n_in, dtype, seed=1)
    check_linear(m, x, m.linear(x))


@pytest.mark.parametrize("tokens", [4, 33, 200])
@pytest.mark.parametrize("group", [32, 128])
def test_strides_and_what_lies_beside_rows_stays(tokens, group):
    m = Matrix(75, 392, group, "bf16", seed=3, apart=1)
    x = rows(tokens, 392, "bf16", seed=4, apart=16)
    wide = torch.full((tokens + 2, 75 + 5), 3.0, dtype=torch.bfloat16, device="cuda")
    add = rows(tokens, 75, "bf16", seed=5, apart=7)
    y = wide[1:-1, 2:77]
    m.linear(x, add, y)
    check_linear(m, x, y, add)
    wide[1:-1, 2:77] = 3.0
    assert (wide == 3.0).all()


@pytest.mark.parametrize("tokens", [1, 20, 130])
def test_residuals_in_place_and_biases(tokens):
    m = Matrix(90, 256, 64, "fp16", seed=6)
    x, y = rows(tokens, 256, "fp16", seed=7), rows(tokens, 90, "fp16", seed=8).contiguous()
    before = y.clone()
    m.linear(x, y, y)
    check_linear(m, x, y, before)
    bias = rows(1, 90, "fp16", seed=9)
    w, out = m.describe(), torch.empty((tokens, 90), dtype=torch.float16, device="cuda")
    need = b.ap_linear_workspace(w, tokens)
    space = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
    b.ap_linear(w, vectors(x), vectors(out), tokens, b.make_vectors(bias.data_ptr(), 90, 0), space.data_ptr(), need, stream_of())
    check_linear(m, x, out, bias.expand(tokens, 90))


@pytest.mark.parametrize("tokens", [1, 16, 50, 150, 400])
def test_what_is_not_a_number_stays_in_its_row(tokens):
    m = Matrix(64, 384, 128, "bf16", seed=10)
    x = rows(tokens, 384, "bf16", seed=11).contiguous()
    clean = m.linear(x).clone()
    x[tokens // 2, 100] = float("nan")
    x[tokens - 1, 5] = float("inf")
    y = m.linear(x)
    odd = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    odd[[tokens // 2, tokens - 1]] = True
    assert torch.equal(y[~odd], clean[~odd])
    assert torch.isnan(y[tokens // 2]).all() and not torch.isfinite(y[tokens - 1]).any()


@pytest.mark.parametrize("tokens", [2, 150])
def test_what_fills_a_block_up_reaches_nothing(tokens):
    """Codes beyond the last column, and values of x beyond it, are whatever they are."""
    m = Matrix(40, 200, 32, "bf16", seed=12)
    x = torch.full((tokens, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :200] = rows(tokens, 200, "bf16", seed=13)
    check_linear(m, x[:, :200], m.linear(x[:, :200]))


@pytest.mark.parametrize("tokens", [8, 300])
def test_weights_of_one_value_and_far_from_zero(tokens):
    m = Matrix(48, 256, 64, "bf16", seed=14)
    m.pairs[:16, :, 0] = 0.0                                   # a step of zero
    m.pairs[16:32, :, 1] = 3.0                                 # a lowest value far above the steps
    x = rows(tokens, 256, "bf16", seed=15)
    check_linear(m, x, m.linear(x))


def test_no_tokens():
    m = Matrix(32, 128, seed=16)
    y = torch.full((1, 32), 5.0, dtype=torch.bfloat16, device="cuda")
    m.linear(rows(1, 128, "bf16"), y=y, n_tokens=0)
    torch.cuda.synchronize()
    assert (y == 5.0).all()


@pytest.mark.parametrize("tokens", [1, 7, 16, 18, 64, 66, 131, 400])
@pytest.mark.parametrize("n_out,n_in,group,dtype,act", [(1, 128, 32, "bf16", "silu"), (50, 264, 64, "fp16", "gelu"), (257, 896, 128, "bf16", "gelu"),
                                                        (160, 2048, 32, "fp16", "silu")])
def test_gated(tokens, n_out, n_in, group, dtype, act):
    gate, up = Matrix(n_out, n_in, group, dtype, seed=20), Matrix(n_out, n_in, group, dtype, seed=21, apart=1)
    x = rows(tokens, n_in, dtype, seed=22, apart=8)
    check_gated(gate, up, x, gated(gate, up, x, act), act)


@pytest.mark.parametrize("tokens", [3, 100])
def test_gates_far_from_zero(tokens):
    """e^-g overflows and the gate is shut, or wide open."""
    gate, up = Matrix(40, 128, 128, "bf16", seed=23), Matrix(40, 128, 128, "bf16", seed=24)
    gate.pairs[:, :, 0] = 0.0
    gate.pairs[:20, :, 1], gate.pairs[20:, :, 1] = 2.0, -2.0
    x = rows(tokens, 128, "bf16", seed=25).abs()
    for act in ("silu", "gelu"):
        h = gated(gate, up, x, act)
        assert torch.isfinite(h).all()
        check_gated(gate, up, x, h, act)


@pytest.mark.parametrize("tokens", [5, 100, 700])
def test_graphs_and_streams(tokens):
    """Captured calls on another stream, replayed with other work between, give what the calls themselves give."""
    m, gate, up = Matrix(200, 1024, 64, seed=30), Matrix(200, 1024, 64, seed=31), Matrix(200, 1024, 64, seed=32)
    x, y, h = rows(tokens, 1024, "bf16", seed=33).contiguous(), *(torch.zeros((tokens, 200), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    need = max(b.ap_linear_workspace(m.describe(), tokens), b.ap_gated_workspace(gate.describe(), up.describe(), tokens), 16)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        m.linear(x, y=y, space=space)
        gated(gate, up, x, h=h, space=space)
    for i in range(4):
        x.copy_(rows(tokens, 1024, "bf16", seed=40 + i))
        y.zero_(), h.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, m.linear(x)) and torch.equal(h, gated(gate, up, x))


@pytest.mark.parametrize("tokens", [1, 64, 300, 1000])
def test_results_are_the_same_each_time(tokens):
    m = Matrix(500, 4096, 128, seed=50)
    x = rows(tokens, 4096, "bf16", seed=51)
    first = m.linear(x)
    for _ in range(3):
        assert torch.equal(first, m.linear(x))


@pytest.mark.parametrize("tokens", [2, 300])
def test_calls_on_two_streams_at_once(tokens):
    ms = [Matrix(300, 2048, 64, seed=60 + i) for i in range(2)]
    xs = [rows(tokens, 2048, "bf16", seed=62 + i) for i in range(2)]
    alone = [m.linear(x) for m, x in zip(ms, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ms]
    out = [torch.zeros((tokens, 300), dtype=torch.bfloat16, device="cuda") for _ in ms]
    spaces = [torch.empty(max(16, b.ap_linear_workspace(m.describe(), tokens)), dtype=torch.uint8, device="cuda") for m in ms]
    torch.cuda.synchronize()
    for _ in range(10):
        for m, x, y, space, s in zip(ms, xs, out, spaces, streams):
            m.linear(x, y=y, stream=s, space=space)
    torch.cuda.synchronize()
    for a, y in zip(alone, out):
        assert torch.equal(a, y)


def test_rows_of_a_matrix_are_a_matrix():
    """A part of the outputs, as a device of several has it, gives the same numbers as the whole."""
    m = Matrix(128, 512, 128, seed=70)
    x = rows(12, 512, "bf16", seed=71)
    whole = m.linear(x)
    part = Matrix(48, 512, 128, seed=70)
    part.words, part.pairs = m.words[32:80], m.pairs[32:80]
    assert torch.equal(part.linear(x), whole[:, 32:80])


def test_far_rows():
    """Rows whose offsets pass 32 bits."""
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GiB of device memory")
    wide = torch.zeros((3, (1 << 30) + 64), dtype=torch.bfloat16, device="cuda")   # 2 GiB apart
    m = Matrix(20, 256, 128, seed=80)
    x = rows(3, 256, "bf16", seed=81)
    wide[:, :256] = x
    y = wide[:, 512:532]
    m.linear(wide[:, :256], y=y)
    check_linear(m, x, y)


@pytest.mark.parametrize("tokens", [1, 4, 5, 8])
@pytest.mark.parametrize("n_in,group,dtype", [(256, 128, "bf16"), (1096, 32, "fp16"), (2056, 64, "bf16")])
def test_outputs_in_several_tiles(tokens, n_in, group, dtype):
    """So many outputs that a workgroup has several tiles of them, of which the last is not full."""
    m = Matrix(256 * 48 + 77, n_in, group, dtype, seed=tokens)
    x = rows(tokens, n_in, dtype, seed=n_in, apart=8)
    check_linear(m, x, m.linear(x))


@pytest.mark.parametrize("tokens", [3, 8, 16])
def test_gated_in_several_tiles(tokens):
    gate, up = (Matrix(256 * 33 + 5, 520, 64, "bf16", seed=90 + i) for i in range(2))
    x = rows(tokens, 520, "bf16", seed=92)
    check_gated(gate, up, x, gated(gate, up, x), "silu")


@pytest.mark.parametrize("tokens", [96, 97, 112, 113, 192, 193, 224, 225, 336, 337])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_tiles_of_tokens(tokens, group):
    """Just full and just overfull tiles of the kernel of many rows."""
    m = Matrix(530, 256, group, "fp16", seed=tokens)
    x = rows(tokens, 256, "fp16", seed=tokens)
    check_linear(m, x, m.linear(x))


@pytest.mark.parametrize("tokens", [120, 3000])
def test_more_outputs_than_one_tile_has_with_many_rows(tokens):
    gate, up = (Matrix(600, 384, 128, "bf16", seed=95 + i) for i in range(2))
    x = rows(tokens, 384, "bf16", seed=97)
    check_gated(gate, up, x, gated(gate, up, x), "silu")


@pytest.mark.parametrize("tokens", [8, 32, 40, 64, 65, 200])
@pytest.mark.parametrize("group", [32, 64])
def test_what_is_not_a_number_stays_in_its_row_with_small_groups(tokens, group):
    m = Matrix(72, 328, group, "fp16", seed=100)
    x = rows(tokens, 328, "fp16", seed=101).contiguous()
    clean = m.linear(x).clone()
    x[tokens // 3, 70], x[tokens - 1, 300] = float("nan"), float("-inf")
    y = m.linear(x)
    odd = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    odd[[tokens // 3, tokens - 1]] = True
    assert torch.equal(y[~odd], clean[~odd])
    assert torch.isnan(y[tokens // 3]).all() and not torch.isfinite(y[tokens - 1]).any()


@pytest.mark.parametrize("tokens", [1, 8, 16, 32, 64, 200])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_a_weight_that_is_not_a_number_reaches_its_output_only(tokens, group):
    m = Matrix(40, 264, group, "bf16", seed=102)
    x = rows(tokens, 264, "bf16", seed=103)
    clean = m.linear(x).clone()
    m.pairs[7, 0, 1], m.pairs[33, 264 // group, 0] = float("nan"), float("nan")
    y = m.linear(x)
    odd = torch.zeros(40, dtype=torch.bool, device="cuda")
    odd[[7, 33]] = True
    assert torch.equal(y[:, ~odd], clean[:, ~odd]) and torch.isnan(y[:, odd]).all()


@pytest.mark.parametrize("tokens", [9, 33, 70, 130])
@pytest.mark.parametrize("n_out,apart,skip", [(516, 0, 0), (516, 1, 0), (516, 4, 1), (516, 4, 2), (516, 4, 4), (514, 2, 4), (513, 0, 3)])
def test_results_at_places_of_any_kind(tokens, n_out, apart, skip):
    """Rows of y and of what is added that begin anywhere and are any distance apart; what lies between them stays."""
    m = Matrix(n_out, 1536, 64, "bf16", seed=110)
    x = rows(tokens, 1536, "bf16", seed=111)
    far = n_out + skip + apart
    space = torch.full((tokens, far), 3.0, dtype=torch.bfloat16, device="cuda")
    before = rows(tokens, far, "bf16", seed=112).contiguous()
    y, add = space[:, skip:skip + n_out], before[:, skip:skip + n_out]
    m.linear(x, add, y)
    check_linear(m, x, y, add)
    assert (space[:, :skip] == 3.0).all() and (space[:, skip + n_out:] == 3.0).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens", [16, 64, 300])
def test_gates_that_are_nearly_shut(tokens, dtype, act):
    """Far below zero what a gate leaves is small, and right relative to its size.

    One weight of 1 a row and one value of x, so g is exact.  With z = g or 2 sqrt(2 / pi) (g + 0.044715 g^3), act = g / (1 + e^-z).  In 32 bits z is
    off by at most 4 2^-24 of itself, so e^z by 4 |z| 2^-24 of itself; by a product and a power of two it is off by (8 + |z|) 2^-23 more, and six
    products and quotients by 2^-24 each.  Powers that 32 bits hold only as less than their least normal number are off by 2^-149."""
    m = Matrix(40, 8, 32, dtype)
    m.pairs[:, :, 0], m.pairs[:, :, 1] = 0.0, 1.0
    x = torch.zeros((tokens, 8), dtype=m.dtype, device="cuda")
    x[:, 0] = -torch.linspace(0.25, 91.0 if act == "silu" else 9.5, tokens, device="cuda")
    g = x[:, 0].double().cpu().numpy()
    z = g if act == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)
    want = g * g / (1.0 + np.exp(-z))                          # up is g too
    u, least = half_step(m.dtype), 2.0 ** -25 if dtype == "fp16" else 2.0 ** -134
    off = np.abs(want) * (4 * np.abs(z) * 2.0 ** -24 + (8 + np.abs(z)) * 2.0 ** -23 + 6 * 2.0 ** -24) + 2.0 ** -148 * np.abs(g)
    got = gated(m, m, x, act).double().cpu().numpy()
    for n in range(40):
        assert (np.abs(got[:, n] - want) <= off * (1 + u) + u * np.abs(want) + least).all()


# Sizes at which a call of few rows takes its inputs in parts: each of the kernel's numbers of tokens, whole and partial last blocks and
# parts, results that go four at a time and that do not.
PARTS = [(20, 514, 4104, 128, "bf16"), (32, 1021, 4352, 32, "fp16"), (17, 72, 6152, 64, "bf16"), (29, 332, 8192, 128, "fp16"), (48, 516, 4232, 64, "bf16"),
         (1, 258, 16392, 128, "bf16"), (4, 65, 20480, 32, "fp16"), (5, 130, 16512, 64, "fp16"), (8, 34, 32776, 128, "bf16"), (16, 516, 16440, 32, "bf16")]
GATED_PARTS = [(1, 514, 8200, 128, "bf16", "silu"), (4, 67, 12296, 32, "fp16", "gelu"), (8, 260, 8192, 64, "bf16", "gelu"), (13, 1030, 8320, 128, "fp16", "silu"),
               (16, 36, 16392, 64, "fp16", "silu"), (20, 130, 8200, 32, "bf16", "gelu"), (32, 258, 8448, 128, "fp16", "silu"), (64, 66, 4104, 64, "bf16", "silu")]


@pytest.mark.parametrize("tokens,n_out,n_in,group,dtype", PARTS)
def test_inputs_in_parts(tokens, n_out, n_in, group, dtype):
    m = Matrix(n_out, n_in, group, dtype, seed=tokens, apart=1)
    assert b.ap_linear_workspace(m.describe(), tokens) >= 2 * 4 * tokens * n_out        # otherwise there are no parts here
    x, add = rows(tokens, n_in, dtype, seed=n_in, apart=8), rows(tokens, n_out, dtype, seed=n_out, apart=3)
    check_linear(m, x, m.linear(x))
    check_linear(m, x, m.linear(x, add), add)


@pytest.mark.parametrize("tokens,n_out,n_in,group,dtype,act", GATED_PARTS)
def test_gated_inputs_in_parts(tokens, n_out, n_in, group, dtype, act):
    gate, up = Matrix(n_out, n_in, group, dtype, seed=tokens), Matrix(n_out, n_in, group, dtype, seed=tokens + 1, apart=1)
    assert b.ap_gated_workspace(gate.describe(), up.describe(), tokens) >= 2 * 8 * tokens * n_out
    x = rows(tokens, n_in, dtype, seed=n_in, apart=8)
    check_gated(gate, up, x, gated(gate, up, x, act), act)


@pytest.mark.parametrize("tokens", [12, 30, 60, 200])
def test_a_share_of_the_outputs_is_the_same_within_roundings(tokens):
    """The order in which a sum's terms are added goes by the sizes of a call and by where in the matrix an output lies: a device's share of
    the outputs, here with more parts and fewer workgroups, is the same product, within what sums in 32 bits may be off."""
    m = Matrix(5000, 4096 + 24, 64, "bf16", seed=71)
    x = rows(tokens, m.n_in, "bf16", seed=72)
    part = Matrix(340, m.n_in, 64, "bf16", seed=71)
    part.words, part.pairs = m.words[3330:3670], m.pairs[3330:3670]
    check_linear(part, x, part.linear(x))
    check_linear(part, x, m.linear(x)[:, 3330:3670])
