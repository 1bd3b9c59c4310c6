"""include/avsg_latent.h, its library symbols and its binding agree, and the
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

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = (("avsg_cache", L.AvsgCache), ("avsg_append", L.AvsgAppend), ("avsg_attention", L.AvsgAttention),
           ("avsg_mx4", L.AvsgMx4))


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "avsg_latent.h")).read(), flags=re.S)


def test_symbols_and_names():
    lib = L.load()
    names = sorted(set(re.findall(r"\b(avsg_[a-z0-9_]+)\s*\(", header())))
    assert len(names) == 9
    for n in names:
        assert hasattr(lib, n) and callable(getattr(L, n)), n
    for n, v in re.findall(r"#define (AVSG_\w+) (\d+)", header()):
        assert getattr(L, n) == int(v), n


def test_struct_layouts(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "avsg_latent.h"', "int main(void) {"]
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


def test_row_bytes():
    assert L.avsg_row_bytes(L.AVSG_ROWS_BF16) == 1152 and L.avsg_row_bytes(L.AVSG_ROWS_MX4) == 400
    assert L.avsg_row_bytes(2) == 0 and L.avsg_row_bytes(-1) == 0


def cache(**kw):
    c = dict(base=4096, pages=8, page_stride=400 * 64, row_stride=400, format=1, batch=2, page_rows=64, pages_per_request=4)
    c.update(kw)
    return L.AvsgCache(**c)


def attention(**kw):
    a = dict(n_q=1, heads=16, topk=64, scale=1.0, d_q=4096, q_token_stride=16 * 576, q_head_stride=576, d_out=8192,
             out_token_stride=16 * 512, out_head_stride=512)
    a.update(kw)
    return L.AvsgAttention(**a)


def append(**kw):
    a = dict(tokens=1, d_latent=4096, latent_stride=512, d_rope=4096, rope_stride=64, d_request=4096, d_position=4096,
             d_angles=4096, positions=1)
    a.update(kw)
    return L.AvsgAppend(**a)


def status(f, *a):
    with pytest.raises(L.AvsgError) as e:
        f(*a)
    assert L.avsg_latent_last_error() in str(e.value) and L.avsg_latent_last_error()
    return e.value.status


@pytest.mark.parametrize("bad,want", [
    (dict(base=0), A.AVSG_E_INVAL), (dict(base=4104), A.AVSG_E_RANGE), (dict(format=3), A.AVSG_E_INVAL),
    (dict(batch=0), A.AVSG_E_INVAL), (dict(pages=0), A.AVSG_E_INVAL), (dict(page_rows=48), A.AVSG_E_NOTPOW2),
    (dict(pages=7), A.AVSG_E_CAPACITY), (dict(row_stride=384), A.AVSG_E_RANGE), (dict(row_stride=408), A.AVSG_E_RANGE),
    (dict(page_stride=400 * 63), A.AVSG_E_RANGE), (dict(format=0), A.AVSG_E_RANGE),
    (dict(pages=2 ** 31), A.AVSG_E_RANGE), (dict(pages_per_request=2 ** 26), A.AVSG_E_RANGE),
    (dict(row_stride=2 ** 60, page_stride=2 ** 62), A.AVSG_E_RANGE)])
def test_caches_refused(bad, want):
    c = cache(**bad)
    assert status(L.avsg_attend, c, attention(), None, 0) == want
    assert status(L.avsg_kv_append, c, append()) == want
    assert status(L.avsg_kv_read, c, 1, 4096, 4096, 4096, 576) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n_q=0), A.AVSG_E_INVAL), (dict(heads=0), A.AVSG_E_INVAL), (dict(topk=-1), A.AVSG_E_INVAL),
    (dict(d_q=0), A.AVSG_E_INVAL), (dict(d_q=4098), A.AVSG_E_INVAL), (dict(q_head_stride=577), A.AVSG_E_INVAL),
    (dict(q_token_stride=4), A.AVSG_E_INVAL), (dict(d_out=0), A.AVSG_E_INVAL), (dict(d_out=8200), A.AVSG_E_INVAL),
    (dict(out_head_stride=513), A.AVSG_E_INVAL), (dict(heads=5000), A.AVSG_E_RANGE), (dict(n_q=2 ** 20), A.AVSG_E_RANGE)])
def test_attentions_refused(bad, want):
    assert status(L.avsg_attend, cache(), attention(**bad), None, 0) == want


def test_workspaces_refused():
    """One request over a long context is shared by several workgroups, whose partial sums need room."""
    need = L.avsg_attend_workspace_bytes(1, 1, 16, 100000)
    big = cache(batch=1, pages=2000, pages_per_request=2000)
    if need:
        assert status(L.avsg_attend, big, attention(topk=100000), None, 0) == A.AVSG_E_INVAL
        assert status(L.avsg_attend, big, attention(topk=100000), 4096, need - 1) == A.AVSG_E_INVAL
        assert status(L.avsg_attend, big, attention(topk=100000), 4097, need) == A.AVSG_E_INVAL
    assert L.avsg_attend_workspace_bytes(0, 1, 16, 64) == 0 and L.avsg_attend_workspace_bytes(1, 1, 16, -1) == 0


@pytest.mark.parametrize("bad,want", [
    (dict(tokens=-1), A.AVSG_E_INVAL), (dict(heads=-1), A.AVSG_E_INVAL), (dict(rope_style=2), A.AVSG_E_INVAL),
    (dict(d_latent=0), A.AVSG_E_INVAL), (dict(d_latent=4100), A.AVSG_E_INVAL), (dict(latent_stride=513), A.AVSG_E_INVAL),
    (dict(d_rope=2), A.AVSG_E_INVAL), (dict(d_request=0), A.AVSG_E_INVAL), (dict(d_position=0), A.AVSG_E_INVAL),
    (dict(d_angles=0), A.AVSG_E_INVAL), (dict(d_angles=4104), A.AVSG_E_INVAL), (dict(positions=-1), A.AVSG_E_INVAL),
    (dict(heads=2), A.AVSG_E_INVAL), (dict(tokens=2 ** 32), A.AVSG_E_RANGE)])
def test_appends_refused(bad, want):
    assert status(L.avsg_kv_append, cache(), append(**bad)) == want


def test_matrices_refused():
    inv, rng = A.AVSG_E_INVAL, A.AVSG_E_RANGE
    q = lambda *a: status(L.avsg_mx4_quantize, *a)  # noqa: E731
    assert q(4096, 2, 1, 32, 32, 4096, 4096) == inv and q(4096, 0, -1, 32, 32, 4096, 4096) == inv
    assert q(4096, 0, 1, 33, 32, 4096, 4096) == rng and q(0, 0, 1, 32, 32, 4096, 4096) == inv
    assert q(4098, 0, 1, 32, 32, 4096, 4096) == inv and q(4096, 0, 2, 32, 36, 4096, 4096) == inv
    assert q(4096, 0, 1, 32, 32, 0, 4096) == inv and q(4096, 0, 1, 32, 32, 4096, 0) == inv
    x = L.AvsgMx4(4096, 4096, 16, 16, 1, 1)
    d = lambda *a: status(L.avsg_mx4_dequantize, *a)  # noqa: E731
    assert d(x, 1, 32, 0, 0, 32) == inv and d(x, 1, 31, 4096, 0, 32) == rng and d(x, 1, 32, 4096, 7, 32) == inv
    assert d(L.AvsgMx4(4096, 4096, 8, 16, 1, 1), 1, 32, 4096, 0, 32) == inv
    m = lambda *a: status(L.avsg_mx4_matmul, *a)  # noqa: E731
    assert m(x, x, 1, 1, 1, 33, 4096, 0, 1, 1) == rng and m(x, x, 1, -1, 1, 32, 4096, 0, 1, 1) == inv
    assert m(x, x, 1, 1, 1, 32, 0, 0, 1, 1) == inv and m(x, x, 1, 1, 1, 32, 4097, 0, 1, 1) == inv
    assert m(x, x, 1, 1, 1, 32, 4096, 3, 1, 1) == inv and m(x, x, 70000, 1, 1, 32, 4096, 0, 1, 1) == rng
    assert m(L.AvsgMx4(4100, 4096, 16, 16, 1, 1), x, 1, 1, 1, 32, 4096, 0, 1, 1) == inv
    assert m(L.AvsgMx4(0, 0, 16, 16, 1, 1), x, 1, 1, 1, 32, 4096, 0, 1, 1) == inv
    assert m(x, x, 1, 2 ** 30, 1, 32, 4096, 0, 1, 1) == rng
