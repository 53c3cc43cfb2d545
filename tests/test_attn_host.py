"""Host side of the cache and attention calls, no GPU: exported symbols, struct layouts as gcc sees them, and every refusal (the
arguments are checked before anything is launched; the addresses here are never followed)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2604_07144_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "autopoiesis_attn.h")
AT = 1 << 20                                               # an address that is aligned and never followed


def _cache(bits=16, **change):
    c = b.make_kv_cache(b.AP_BF16, bits, 10, 16, 2, 128, AT, AT, AT if bits == 4 else 0, AT if bits == 4 else 0)
    for f, x in change.items():
        setattr(c, f, x)
    return c


def _batch(**change):
    x = b.make_seq_batch(3, 3, 1, 100, AT, AT, AT, 7)
    for f, y in change.items():
        setattr(x, f, y)
    return x


def _rows(**change):
    x = b.make_rows(AT, 8, 128)
    for f, y in change.items():
        setattr(x, f, y)
    return x


def test_every_declared_symbol_is_exported():
    names = re.findall(r"\b(ap_\w+)\(", re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S))
    assert sorted(set(names)) == ["ap_attention", "ap_attention_workspace", "ap_kv_append", "ap_kv_read"]
    for n in names:
        getattr(b.lib(), n)


def test_struct_layouts_match_the_header_as_gcc_sees_it(tmp_path):
    structs = {"ap_kv_cache": b.ApKvCache, "ap_seq_batch": b.ApSeqBatch, "ap_rows": b.ApRows, "ap_rotation": b.ApRotation}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "autopoiesis_attn.h"', "int main(void) {"]
    for name, t in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in t._fields_]
    (tmp_path / "s.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "s.c", "-o", "s"], cwd=tmp_path, check=True)
    got = dict(line.split() for line in subprocess.run(["./s"], cwd=tmp_path, check=True, capture_output=True, text=True).stdout.splitlines())
    for name, t in structs.items():
        assert int(got[name]) == ctypes.sizeof(t)
        for f, _ in t._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(t, f).offset, (name, f)


def _refused(status, call, *args):
    with pytest.raises(b.ApError) as e:
        call(*args)
    assert e.value.status == status, args


BAD_CACHE = [dict(dtype=2), dict(bits=8), dict(head_dim=96), dict(head_dim=0), dict(n_pages=0), dict(page_size=0), dict(kv_heads=0), dict(k=None),
             dict(v=None), dict(k=AT + 8), dict(v=AT + 2), dict(page_stride=-16), dict(head_stride=8), dict(slot_stride=40)]
BAD_PAIRS = [dict(k_pairs=None), dict(v_pairs=AT + 4), dict(pair_page_stride=4), dict(pair_slot_stride=-8), dict(pair_head_stride=2)]
BAD_BATCH = [dict(n_seqs=0), dict(max_kv=0), dict(max_new=0), dict(table_width=0), dict(new_first=None), dict(kv_len=None), dict(page_table=None),
             dict(table_stride=6), dict(kv_len=AT + 2)]
LONG_BATCH = [dict(max_kv=7 * 16 + 1), dict(n_tokens=1 << 31), dict(n_seqs=1 << 31, n_tokens=1)]
BAD_ROWS = [dict(data=None), dict(data=AT + 2), dict(token_stride=8), dict(head_stride=-256)]


def _calls(cache=None, batch=None, rows=None):
    c, x, r = cache or _cache(), batch or _batch(), rows or _rows()
    yield b.ap_kv_append, (c, x, r, _rows())
    yield b.ap_kv_append, (c, x, _rows(), r)
    yield b.ap_kv_append, (c, x, _rows(), _rows(), None, r, _rows(), 8)
    yield b.ap_kv_append, (c, x, _rows(), _rows(), None, _rows(), r, 8)
    yield b.ap_kv_read, (c, x, r, _rows())
    yield b.ap_kv_read, (c, x, _rows(), r)
    yield b.ap_attention, (c, x, r, _rows(), 8, 0.1, 0, 0, AT, 1 << 40)
    yield b.ap_attention, (c, x, _rows(), r, 8, 0.1, 0, 0, AT, 1 << 40)


@pytest.mark.parametrize("change", BAD_CACHE)
def test_caches_that_are_refused(change):
    for call, args in _calls(cache=_cache(**change)):
        _refused(b.AP_ERR_INVALID, call, *args)
    _refused(b.AP_ERR_INVALID, b.ap_attention_workspace, _cache(**change), _batch(), 8)


@pytest.mark.parametrize("change", BAD_PAIRS)
def test_pairs_that_are_refused(change):
    for call, args in _calls(cache=_cache(4, **change)):
        _refused(b.AP_ERR_INVALID, call, *args)


@pytest.mark.parametrize("change", BAD_BATCH)
def test_batches_that_are_refused(change):
    for call, args in _calls(batch=_batch(**change)):
        _refused(b.AP_ERR_INVALID, call, *args)
    _refused(b.AP_ERR_INVALID, b.ap_attention_workspace, _cache(), _batch(**change), 8)


@pytest.mark.parametrize("change", LONG_BATCH)
def test_batches_that_are_too_long(change):
    for call, args in _calls(batch=_batch(**change)):
        _refused(b.AP_ERR_RANGE, call, *args)


@pytest.mark.parametrize("change", BAD_ROWS)
def test_rows_that_are_refused(change):
    for call, args in _calls(rows=_rows(**change)):
        if any(isinstance(a, b.ApRows) and any(getattr(a, f) == x for f, x in change.items()) for a in args):
            _refused(b.AP_ERR_INVALID, call, *args)


def test_rotations_that_are_refused():
    for status, turn in ((b.AP_ERR_INVALID, b.make_rotation(0, 100, 64)), (b.AP_ERR_INVALID, b.make_rotation(AT + 4, 100, 64)),
                         (b.AP_ERR_INVALID, b.make_rotation(AT, 100, 0)), (b.AP_ERR_INVALID, b.make_rotation(AT, 100, 24)),
                         (b.AP_ERR_INVALID, b.make_rotation(AT, 100, 144)), (b.AP_ERR_RANGE, b.make_rotation(AT, 99, 64))):
        _refused(status, b.ap_kv_append, _cache(), _batch(), _rows(), _rows(), turn)
    _refused(b.AP_ERR_INVALID, b.ap_kv_append, _cache(), _batch(), _rows(), _rows(), None, _rows(), _rows(), 0)
    _refused(b.AP_ERR_INVALID, b.ap_kv_append, _cache(), _batch(), _rows(), _rows(), None, _rows(), None, 8)


def test_arguments_of_attention_that_are_refused():
    for heads, scale in ((0, 0.1), (7, 0.1), (8, 0.0), (8, -1.0), (8, float("nan")), (8, float("inf"))):
        _refused(b.AP_ERR_INVALID, b.ap_attention, _cache(), _batch(), _rows(), _rows(), heads, scale, 0, 0, AT, 1 << 40)
    _refused(b.AP_ERR_INVALID, b.ap_attention_workspace, _cache(), _batch(), 7)
    _refused(b.AP_ERR_RANGE, b.ap_attention_workspace, _cache(), _batch(n_tokens=1 << 28), 8)
    batch = _batch(max_kv=5000, table_width=400, table_stride=400)
    need = b.ap_attention_workspace(_cache(), batch, 8)
    assert need > 0
    for space, size in ((0, need), (AT, need - 1), (AT + 8, need)):
        _refused(b.AP_ERR_INVALID, b.ap_attention, _cache(), batch, _rows(), _rows(), 8, 0.1, 0, 0, space, size)
    assert b.lib().ap_attention_workspace(_cache(), batch, 8, 0, 0, None) == b.AP_ERR_INVALID


def test_no_new_tokens_is_no_work():
    empty = _batch(n_tokens=0, max_new=0)
    b.ap_kv_append(_cache(), empty, _rows(), _rows())
    b.ap_kv_read(_cache(), empty, _rows(), _rows())
    assert b.ap_attention_workspace(_cache(), empty, 8) == 0
    b.ap_attention(_cache(), empty, _rows(), _rows(), 8, 0.1)


def test_workspaces_do_not_grow_with_the_length():
    batch = lambda n, m: b.make_seq_batch(3, 3 * m, m, n, AT, AT, AT, -(-n // 16))   # noqa: E731
    assert b.ap_attention_workspace(_cache(), batch(100, 1), 8) == 0                 # short sequences are not split
    long = b.ap_attention_workspace(_cache(), batch(1 << 20, 1), 8)
    assert 0 < long == b.ap_attention_workspace(_cache(), batch(1 << 22, 1), 8)      # pieces are as many as wavefronts
    assert b.ap_attention_workspace(_cache(), batch(1 << 20, 1), 8, 100, 4) == 0     # a window makes them short
    whole = b.make_seq_batch(1, 16384, 16384, 1 << 20, AT, AT, AT, 1 << 16)
    assert b.ap_attention_workspace(_cache(), whole, 8) == 0                         # many rows: enough work without a split


def test_scales_beyond_what_scores_are_held_in():
    """Scores are held in powers of two, so a scale is refused where log2(e) times it is no number of 32 bits."""
    for scale in (2.4e38, 3e38):
        _refused(b.AP_ERR_INVALID, b.ap_attention, _cache(), _batch(), _rows(), _rows(), 8, scale, 0, 0, AT, 1 << 40)
    b.ap_attention(_cache(), _batch(n_tokens=0, max_new=0), _rows(), _rows(), 8, 2.3e38)
