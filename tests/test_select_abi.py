"""include/avsg_select.h, its library symbols and its binding agree, and the
host-side checks refuse what the kernels cannot take (no GPU needed: a refused
call enqueues nothing)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_37538_amd import avsg as A
from paper_2609_37538_amd import latent as L
from paper_2609_37538_amd import selection as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = (("avsg_key_cache", S.AvsgKeyCache), ("avsg_key_append", S.AvsgKeyAppend), ("avsg_selection", S.AvsgSelection))


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "avsg_select.h")).read(), flags=re.S)


def test_symbols_and_names():
    lib = S.load()
    names = sorted(set(re.findall(r"\b(avsg_[a-z0-9_]+)\s*\(", header())))
    assert len(names) == 5
    for n in names:
        assert hasattr(lib, n) and callable(getattr(S, n)), n
    for n, v in re.findall(r"#define (AVSG_\w+) (\d+)", header()):
        assert getattr(S, n) == int(v), n


def test_struct_layouts(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "avsg_select.h"', "int main(void) {"]
    for name, py in STRUCTS:
        lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'printf("{name} {f} %zu\\n", offsetof({name}, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;", "}"]) + "\n")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    got = {tuple(s.split()[:2]): int(s.split()[2]) for s in said if s}
    for name, py in STRUCTS:
        assert got[(name, "size")] == ctypes.sizeof(py), name
        for f, _ in py._fields_:
            assert got[(name, f)] == getattr(py, f).offset, f"{name}.{f}"


def cache(**kw):
    c = dict(base=4096, pages=8, page_stride=132 * 64, row_stride=132, batch=2, page_rows=64, pages_per_request=4)
    c.update(kw)
    return S.AvsgKeyCache(**c)


def selection(**kw):
    a = dict(n_q=1, heads=16, longest=256, topk=64, block=1, first=0, recent=0, d_q=4096, q_token_stride=16 * 128,
             q_head_stride=128, d_weights=4096, weight_stride=16, d_index=4096)
    a.update(kw)
    return S.AvsgSelection(**a)


def append(**kw):
    a = dict(tokens=1, d_key=4096, key_stride=128, d_request=4096, d_position=4096, d_angles=4096, positions=1)
    a.update(kw)
    return S.AvsgKeyAppend(**a)


def status(f, *a):
    with pytest.raises(L.AvsgError) as e:
        f(*a)
    assert L.avsg_latent_last_error() in str(e.value) and L.avsg_latent_last_error()
    return e.value.status


@pytest.mark.parametrize("bad,want", [
    (dict(base=0), A.AVSG_E_INVAL), (dict(base=4098), A.AVSG_E_RANGE), (dict(batch=0), A.AVSG_E_INVAL),
    (dict(pages=0), A.AVSG_E_INVAL), (dict(page_rows=48), A.AVSG_E_NOTPOW2), (dict(pages=7), A.AVSG_E_CAPACITY),
    (dict(row_stride=128), A.AVSG_E_RANGE), (dict(row_stride=134), A.AVSG_E_RANGE), (dict(page_stride=132 * 63), A.AVSG_E_RANGE),
    (dict(pages=2 ** 31), A.AVSG_E_RANGE), (dict(pages_per_request=2 ** 26), A.AVSG_E_RANGE),
    (dict(row_stride=2 ** 60, page_stride=2 ** 62), A.AVSG_E_RANGE)])
def test_caches_refused(bad, want):
    c = cache(**bad)
    assert status(S.avsg_select, c, selection(), 4096, 1 << 20) == want
    assert status(S.avsg_key_append_rows, c, append()) == want
    assert status(S.avsg_key_read_rows, c, 1, 4096, 4096, 4096, 128) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n_q=0), A.AVSG_E_INVAL), (dict(heads=0), A.AVSG_E_INVAL), (dict(heads=129), A.AVSG_E_RANGE),
    (dict(topk=-1), A.AVSG_E_INVAL), (dict(longest=-4), A.AVSG_E_INVAL), (dict(topk=257), A.AVSG_E_RANGE),
    (dict(longest=257), A.AVSG_E_CAPACITY), (dict(block=0), A.AVSG_E_NOTPOW2), (dict(block=3), A.AVSG_E_NOTPOW2),
    (dict(block=256), A.AVSG_E_NOTPOW2), (dict(block=128, topk=64), A.AVSG_E_RANGE), (dict(block=16, longest=250, topk=64), A.AVSG_E_RANGE),
    (dict(first=-1), A.AVSG_E_INVAL), (dict(recent=-1), A.AVSG_E_INVAL), (dict(d_q=0), A.AVSG_E_INVAL), (dict(d_q=4104), A.AVSG_E_INVAL),
    (dict(q_head_stride=120), A.AVSG_E_INVAL), (dict(q_token_stride=8), A.AVSG_E_INVAL), (dict(d_weights=0), A.AVSG_E_INVAL),
    (dict(d_weights=4097), A.AVSG_E_INVAL), (dict(d_index=0), A.AVSG_E_INVAL), (dict(d_scores=4098), A.AVSG_E_INVAL),
    (dict(n_q=2 ** 19), A.AVSG_E_RANGE), (dict(longest=2 ** 30 + 1), A.AVSG_E_RANGE)])
def test_selections_refused(bad, want):
    assert status(S.avsg_select, cache(), selection(**bad), 4096, 1 << 20) == want


def test_workspaces():
    least = S.avsg_select_workspace_least(256, 1)
    assert least == 1024 and S.avsg_select_workspace_least(1000 * 8, 8) == 4000 and S.avsg_select_workspace_least(1001, 1) == 4016
    for at, size in ((None, 1 << 20), (4104, 1 << 20), (4096, least - 1), (4096, 0)):
        assert status(S.avsg_select, cache(), selection(), at, size) == A.AVSG_E_INVAL
    assert S.avsg_select_workspace_bytes(2, 3, 256, 1) == 6 * 1024
    assert S.avsg_select_workspace_bytes(64, 4096, 131072, 1) == 128 << 20
    assert S.avsg_select_workspace_bytes(1, 1, 2 ** 30, 1) == 2 ** 32      # never less than a token's
    for bad in ((0, 1, 256, 1), (1, 0, 256, 1), (1, 1, 0, 1), (1, 1, 256, 3), (1, 1, 250, 4)):
        assert S.avsg_select_workspace_bytes(*bad) == 0
    assert S.avsg_select_workspace_least(2 ** 30 + 1, 1) == 0 and S.avsg_select_workspace_least(-1, 1) == 0 and S.avsg_select_workspace_least(256, 256) == 0


def test_empty_calls_take_nothing():
    S.avsg_select(cache(), selection(topk=0, d_q=0, d_index=0), None, 0)
    S.avsg_key_append_rows(cache(), append(tokens=0, d_key=0))
    S.avsg_key_read_rows(cache(), 0, 0, 0, 0, 0)


@pytest.mark.parametrize("bad,want", [
    (dict(tokens=-1), A.AVSG_E_INVAL), (dict(heads=-1), A.AVSG_E_INVAL), (dict(positions=-1), A.AVSG_E_INVAL),
    (dict(rope_style=2), A.AVSG_E_INVAL), (dict(rope_at=32), A.AVSG_E_INVAL), (dict(rope_at=-2), A.AVSG_E_INVAL),
    (dict(d_key=0), A.AVSG_E_INVAL), (dict(d_key=4100), A.AVSG_E_INVAL), (dict(key_stride=129), A.AVSG_E_INVAL),
    (dict(d_request=0), A.AVSG_E_INVAL), (dict(d_position=0), A.AVSG_E_INVAL), (dict(d_angles=0), A.AVSG_E_INVAL),
    (dict(d_angles=4104), A.AVSG_E_INVAL), (dict(tokens=2 ** 28), A.AVSG_E_RANGE), (dict(heads=2), A.AVSG_E_INVAL),
    (dict(heads=2, d_q=4096, q_head_stride=128, d_q_out=4096, q_out_head_stride=128), A.AVSG_E_INVAL),
    (dict(heads=2, d_q=4096, q_head_stride=128, d_q_out=4104, q_out_head_stride=128, d_weights_out=4096), A.AVSG_E_INVAL),
    (dict(heads=2, d_q=4096, q_head_stride=128, d_q_out=4096, q_out_head_stride=120, d_weights_out=4096), A.AVSG_E_INVAL),
    (dict(heads=2, d_q=4096, q_head_stride=100, d_q_out=4096, q_out_head_stride=128, d_weights_out=4096), A.AVSG_E_INVAL),
    (dict(heads=2, d_q=4096, q_head_stride=128, d_q_out=4096, q_out_head_stride=128, d_weights_out=4096, d_weights=4097), A.AVSG_E_INVAL),
    (dict(tokens=2 ** 20, heads=2 ** 20, d_q=4096, q_head_stride=128, d_q_out=4096, q_out_head_stride=128, d_weights_out=4096), A.AVSG_E_RANGE)])
def test_appends_refused(bad, want):
    assert status(S.avsg_key_append_rows, cache(), append(**bad)) == want


def test_reads_refused():
    inv = A.AVSG_E_INVAL
    read = lambda *a: status(S.avsg_key_read_rows, cache(), *a)  # noqa: E731
    assert read(-1, 4096, 4096, 4096, 128) == inv and read(1, 0, 4096, 4096, 128) == inv and read(1, 4096, 0, 4096, 128) == inv
    assert read(1, 4096, 4096, 0, 128) == inv and read(1, 4096, 4096, 4100, 128) == inv and read(1, 4096, 4096, 4096, 130) == inv
    assert read(2 ** 28, 4096, 4096, 4096, 128) == A.AVSG_E_RANGE
