"""Host side of the calls on weights in 4 bits and of log probabilities, no GPU: exported symbols, struct layouts as gcc sees them, and
every refusal (the arguments are checked before anything is launched; the addresses here are never followed)."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import linear as orc
from paper_2604_07144_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "autopoiesis_linear.h")
AT = 1 << 20                                               # an address that is aligned and never followed


def _made(x, change):
    for f, y in change.items():
        setattr(x, f, y)
    return x


def _weights(**change):
    return _made(b.make_weights(b.AP_BF16, 128, 100, 264, AT, AT), change)


def _rows(**change):
    return _made(b.make_vectors(AT, 264), change)


def _logits(**change):
    return _made(b.make_logits(b.AP_BF16, 5, 1000, AT), change)


def _refused(status, call, *args):
    with pytest.raises(b.ApError) as e:
        call(*args)
    assert e.value.status == status, args


def test_every_declared_symbol_is_exported():
    names = re.findall(r"\b(ap_\w+)\(", re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S))
    assert sorted(set(names)) == ["ap_gated", "ap_gated_workspace", "ap_linear", "ap_linear_workspace", "ap_logprobs", "ap_logprobs_workspace",
                                  "ap_weights_pack", "ap_weights_read"]
    for n in names:
        getattr(b.lib(), n)


def test_struct_layouts_match_the_header_as_gcc_sees_it(tmp_path):
    structs = {"ap_weights": b.ApWeights, "ap_vectors": b.ApVectors, "ap_logits": b.ApLogits}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "autopoiesis_linear.h"', "int main(void) {"]
    for name, t in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
    lines.append('printf("AP_FP32 %u\\nAP_SILU %u\\nAP_GELU %u\\n", AP_FP32, AP_SILU, AP_GELU);')
    (tmp_path / "s.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "s.c", "-o", "s"], cwd=tmp_path, check=True)
    got = dict(line.split() for line in subprocess.run(["./s"], cwd=tmp_path, check=True, capture_output=True, text=True).stdout.splitlines())
    for name, t in structs.items():
        assert int(got[name]) == ctypes.sizeof(t)
        for f, _ in t._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(t, f).offset, (name, f)
    for n in ("AP_FP32", "AP_SILU", "AP_GELU"):
        assert int(got[n]) == getattr(b, n)


def _calls(w, x=None, y=None):
    x, y = x or _rows(), y or _rows()
    yield b.ap_weights_pack, (w, x)
    yield b.ap_weights_read, (w, x)
    yield b.ap_linear, (w, x, y, 3, None, AT, 1 << 40)
    yield b.ap_gated, (w, _weights(), x, y, 3, b.AP_SILU, AT, 1 << 40)
    yield b.ap_gated, (_weights(), w, x, y, 3, b.AP_SILU, AT, 1 << 40)


BAD_WEIGHTS = [dict(dtype=2), dict(group=16), dict(group=0), dict(group=96), dict(n_out=0), dict(n_in=0), dict(n_in=260), dict(codes=None), dict(pairs=None),
               dict(codes=AT + 8), dict(pairs=AT + 2), dict(code_stride=-64), dict(code_stride=200), dict(pair_stride=6), dict(pair_stride=-4)]


@pytest.mark.parametrize("change", BAD_WEIGHTS)
def test_weights_that_are_refused(change):
    for call, args in _calls(_weights(**change)):
        _refused(b.AP_ERR_INVALID, call, *args)
    _refused(b.AP_ERR_INVALID, b.ap_linear_workspace, _weights(**change), 3)
    _refused(b.AP_ERR_INVALID, b.ap_gated_workspace, _weights(**change), _weights(), 3)
    _refused(b.AP_ERR_INVALID, b.ap_gated_workspace, _weights(), _weights(**change), 3)


def test_pairs_of_a_block_are_aligned():
    for group, good in ((128, 4), (64, 8), (32, 16)):
        w = b.make_weights(b.AP_BF16, group, 10, 128, AT, AT + good)
        assert b.ap_linear_workspace(w, 0) == 0
        _refused(b.AP_ERR_INVALID, b.ap_linear_workspace, _made(w, dict(pairs=AT + good // 2)), 3)


@pytest.mark.parametrize("change", [dict(n_out=1 << 31), dict(n_in=1 << 31), dict(n_out=1 << 22, n_in=1 << 20)])
def test_weights_that_are_too_large(change):
    for call, args in _calls(_weights(**change)):
        _refused(b.AP_ERR_RANGE, call, *args)


@pytest.mark.parametrize("change", [dict(data=None), dict(data=AT + 8), dict(stride=8), dict(stride=-528)])
def test_rows_that_are_refused(change):
    for call, args in _calls(_weights(), x=_rows(**change)):
        _refused(b.AP_ERR_INVALID, call, *args)


@pytest.mark.parametrize("change", [dict(data=None), dict(data=AT + 1), dict(stride=3), dict(stride=-2)])
def test_results_that_are_refused(change):
    bad = _rows(**change)
    _refused(b.AP_ERR_INVALID, b.ap_linear, _weights(), _rows(), bad, 3, None, AT, 1 << 40)
    _refused(b.AP_ERR_INVALID, b.ap_linear, _weights(), _rows(), _rows(), 3, bad, AT, 1 << 40)
    _refused(b.AP_ERR_INVALID, b.ap_gated, _weights(), _weights(), _rows(), bad, 3, b.AP_SILU, AT, 1 << 40)


def test_arguments_of_products_that_are_refused():
    _refused(b.AP_ERR_INVALID, b.ap_gated, _weights(), _weights(), _rows(), _rows(), 3, 2, AT, 1 << 40)
    for other in (dict(dtype=b.AP_FP16), dict(group=64, pairs=AT, pair_stride=24), dict(n_out=99), dict(n_in=256)):
        _refused(b.AP_ERR_INVALID, b.ap_gated, _weights(), _weights(**other), _rows(), _rows(), 3, b.AP_SILU, AT, 1 << 40)
        _refused(b.AP_ERR_INVALID, b.ap_gated_workspace, _weights(), _weights(**other), 3)
    _refused(b.AP_ERR_RANGE, b.ap_linear, _weights(), _rows(), _rows(), 1 << 31, None, AT, 1 << 40)
    _refused(b.AP_ERR_RANGE, b.ap_linear_workspace, _weights(), (1 << 32) - 1)
    assert b.lib().ap_linear_workspace(_weights(), 3, None) == b.AP_ERR_INVALID
    assert b.lib().ap_gated_workspace(_weights(), _weights(), 3, None) == b.AP_ERR_INVALID


@pytest.mark.parametrize("tokens", [64, 100, 300, 1000, 5000])
def test_workspaces_that_are_refused(tokens):
    """Where a workspace is needed it has to be there, aligned and large enough."""
    w = b.make_weights(b.AP_BF16, 128, 4096, 14336, AT, AT)
    x, y = b.make_vectors(AT, 14336), b.make_vectors(AT, 4096)
    for need, call in ((b.ap_linear_workspace(w, tokens), lambda at, n: b.ap_linear(w, x, y, tokens, None, at, n)),
                       (b.ap_gated_workspace(w, w, tokens), lambda at, n: b.ap_gated(w, w, x, y, tokens, b.AP_SILU, at, n))):
        if need:
            for at, n in ((0, need), (AT, need - 1), (AT + 8, need)):
                _refused(b.AP_ERR_INVALID, call, at, n)


def test_no_tokens_are_no_work():
    b.ap_linear(_weights(), _rows(), _rows(), 0)
    b.ap_gated(_weights(), _weights(), _rows(), _rows(), 0)
    assert b.ap_linear_workspace(_weights(), 0) == b.ap_gated_workspace(_weights(), _weights(), 0) == 0
    b.ap_logprobs(_logits(n_rows=0), AT, 1.0, 5, AT, AT, AT, AT)
    assert b.ap_logprobs_workspace(_logits(n_rows=0), 64) == 0


@pytest.mark.parametrize("change", [dict(dtype=3), dict(vocab=0), dict(data=None), dict(data=AT + 1), dict(stride=-2000), dict(stride=2001),
                                    dict(dtype=b.AP_FP32, stride=2), dict(dtype=b.AP_FP32, stride=4000, data=AT + 2)])
def test_logits_that_are_refused(change):
    _refused(b.AP_ERR_INVALID, b.ap_logprobs, _logits(**change), AT, 1.0, 5, AT, AT, AT, AT, AT, 1 << 40)
    _refused(b.AP_ERR_INVALID, b.ap_logprobs_workspace, _logits(**change), 5)


def test_arguments_of_log_probabilities_that_are_refused():
    good = [AT, 1.0, 5, AT, AT, AT, AT, AT, 1 << 40]
    for at, bad in ((1, 0.0), (1, -1.0), (1, float("nan")), (1, float("inf")), (1, 3e38), (2, 65), (0, 0), (3, 0), (5, 0), (6, 0), (0, AT + 2), (3, AT + 1),
                    (4, AT + 2), (5, AT + 2), (6, AT + 3)):
        args = list(good)
        args[at] = bad
        _refused(b.AP_ERR_INVALID, b.ap_logprobs, _logits(), *args)
    assert b.lib().ap_logprobs_workspace(_logits(), 5, None) == b.AP_ERR_INVALID
    for change in (dict(vocab=1 << 31), dict(n_rows=1 << 31)):
        _refused(b.AP_ERR_RANGE, b.ap_logprobs, _logits(**change), *good)
    long = _logits(vocab=128256, stride=2 * 128256)
    need = b.ap_logprobs_workspace(long, 5)
    assert need > 0
    for at, n in ((0, need), (AT, need - 1), (AT + 8, need)):
        _refused(b.AP_ERR_INVALID, b.ap_logprobs, long, AT, 1.0, 5, AT, AT, AT, AT, at, n)


def test_rows_of_weights_in_bytes():
    assert b.weight_row_bytes(128, 128) == (64, 4) and b.weight_row_bytes(32, 136) == (128, 32) and b.weight_row_bytes(64, 4096) == (2048, 256)


def test_every_code_has_a_place_of_its_own():
    seen = {orc.place(c) for c in range(256)}
    assert len(seen) == 256 and {w for w, _ in seen} == set(range(32)) and {s for _, s in seen} == set(range(0, 32, 4))
    words = np.zeros((1, 16), np.uint32)
    words[0, orc.place(77)[0]] = np.uint32(11) << np.uint32(orc.place(77)[1])
    assert np.nonzero(orc.values(words, np.array([[[1.0, 0.0]]]), 128, 128)[0])[0].tolist() == [77]


@pytest.mark.parametrize("scale", [2.0 ** -121, 1e-38, 1e-45])
def test_scales_that_are_too_small(scale):
    """Below 2^-120 (times log2(e)) logits in 32 bits could be further apart than 32 bits hold, and yet both count."""
    _refused(b.AP_ERR_INVALID, b.ap_logprobs, _logits(dtype=b.AP_FP32, stride=4000), AT, scale, 5, AT, AT, AT, AT, AT, 1 << 40)
    b.ap_logprobs(_logits(n_rows=0), AT, 2.0 ** -120, 5, AT, AT, AT, AT)


def test_rows_that_are_written_do_not_overlap():
    """What two rows write to one place would go by timing."""
    args = (AT, 1 << 40)
    for stride in (0, 198):                                # of 100 outputs
        y = _rows(stride=stride)
        _refused(b.AP_ERR_INVALID, b.ap_linear, _weights(), _rows(), y, 3, None, *args)
        _refused(b.AP_ERR_INVALID, b.ap_gated, _weights(), _weights(), _rows(), y, 3, b.AP_SILU, *args)
        b.ap_linear(_weights(), _rows(), y, 0, None, *args)
        b.ap_gated(_weights(), _weights(), _rows(), y, 0, b.AP_SILU, *args)
    for change in (dict(code_stride=0), dict(code_stride=176), dict(pair_stride=0), dict(pair_stride=8)):
        _refused(b.AP_ERR_INVALID, b.ap_weights_pack, _weights(**change), _rows())
        assert b.ap_linear_workspace(_weights(**change), 3) == 0          # rows that are read may
    for stride in (0, 512):
        _refused(b.AP_ERR_INVALID, b.ap_weights_read, _weights(), _rows(stride=stride))


def test_a_workspace_is_for_one_number_of_tokens():
    """Many tokens fill the chip without parts, a few hundred do not: a buffer for the most of them is refused for fewer."""
    w, x, y = b.make_weights(b.AP_BF16, 128, 4096, 14336, AT, AT), b.make_vectors(AT, 14336), b.make_vectors(AT, 4096)
    needs = {n: b.ap_linear_workspace(w, n) for n in (300, 8192)}
    assert needs[8192] < needs[300]
    _refused(b.AP_ERR_INVALID, b.ap_linear, w, x, y, 300, None, AT, needs[8192])
