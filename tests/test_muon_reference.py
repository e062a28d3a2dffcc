"""The Muon direction's 64-bit reference against singular values, and what the entry point refuses (no GPU)."""
import ctypes
import os
import subprocess

import pytest
import torch

import _muon as M
import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import _build

BAD = P.PURO_ERR_INVALID_ARG
A = 0x100000  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return P.load_library()


@pytest.mark.parametrize("r,c", [(1, 1), (5, 9), (9, 5), (24, 24), (7, 40)])
def test_the_definition_maps_singular_values(r, c):
    v = M.gradient(r, c, 1)
    p, s, q = torch.linalg.svd(v.double(), full_matrices=False)
    want = p @ torch.diag(M.singular_value(s / s.norm())) @ q
    assert (M.exact(v) - want).norm() <= 1e-12 * want.norm() * (r + c)


def test_the_model_differs_by_roundings_only():
    for r, c, low, high in ((40, 70, 1e-5, 2e-2), (20, 70, 1e-8, 1e-4), (70, 20, 1e-8, 1e-4)):  # FP16's, and with all digits
        v = M.gradient(r, c, 3, "noise")
        assert low < (M.model(v) - M.exact(v)).norm() / M.exact(v).norm() < high


def entry(grad=A, momentum=A, u=A, rows=64, cols=96, gs=96, us=96, gt=0, ut=1, reserved=0):
    return P.puro_muon_matrix_t(grad, momentum, u, rows, cols, gs, us, gt, ut, reserved)


def table(*entries):
    t = (P.puro_muon_matrix_t * max(1, len(entries)))(*entries)
    t.count = len(entries)
    return t


def call(lib, t, momentum=0.95, coefficients=M.STEPS, steps=None, ws=A, ws_bytes=1 << 40, status=None):
    flat = [x for s in coefficients for x in s]
    return lib.puro_muon_direction_grouped(t, t.count, momentum, 1, (ctypes.c_double * max(1, len(flat)))(*flat),
                                           len(coefficients) if steps is None else steps, ws, ws_bytes, status, None)


def test_malformed_matrices_are_refused(lib):
    good = entry()
    for bad in (dict(grad=None), dict(u=None), dict(grad=A + 1), dict(momentum=A + 2), dict(u=A + 2), dict(rows=-1), dict(cols=-3),
                dict(gs=-96), dict(us=95), dict(gt=2), dict(ut=-1), dict(reserved=1), dict(gt=1, grad=A + 2)):
        t = table(good, entry(**bad))
        assert call(lib, t) == BAD, bad
        assert lib.puro_muon_direction_workspace_size(t, 2) == 0
    for big in (dict(rows=(1 << 20) + 1), dict(cols=1 << 21, gs=1 << 21, us=1 << 21)):
        assert call(lib, table(entry(**big))) == P.PURO_ERR_UNSUPPORTED


def test_malformed_calls_are_refused(lib):
    t = table(entry(), entry(rows=200))
    nan, inf = float("nan"), float("inf")
    need = lib.puro_muon_direction_workspace_size(t, 2)
    assert need > 8 * (64 * 96 + 96 * 200)
    for kw in (dict(momentum=-0.1), dict(momentum=1.5), dict(momentum=nan), dict(steps=0), dict(steps=-1), dict(steps=65), dict(ws=None),
               dict(ws=A + 16), dict(ws_bytes=need - 1), dict(status=A + 2), dict(coefficients=((nan, 0, 0),)), dict(coefficients=((1, inf, 0),)),
               dict(coefficients=((2000, 0, 0),)), dict(coefficients=((30.0, 0, 0),) * 3)):
        assert call(lib, t, **kw) == BAD, kw
    assert lib.puro_muon_direction_grouped(None, 1, 0.5, 0, (ctypes.c_double * 3)(1, 0, 0), 1, A, 1 << 40, None, None) == BAD
    assert lib.puro_muon_direction_grouped(t, -1, 0.5, 0, (ctypes.c_double * 3)(1, 0, 0), 1, A, 1 << 40, None, None) == BAD
    assert lib.puro_muon_direction_grouped(t, 2, 0.5, 0, None, 1, A, 1 << 40, None, None) == BAD


def test_nothing_to_do(lib):
    assert call(lib, table(), ws=None, ws_bytes=0) == P.PURO_OK
    assert call(lib, table(entry(rows=0, grad=None, u=None), entry(cols=0, gs=0, us=0)), ws=None, ws_bytes=0) == P.PURO_OK


def test_scratch_is_of_the_largest_launch(lib):
    """Many matrices take turns with the scratch of 128; few shapes or many."""
    one = lib.puro_muon_direction_workspace_size(table(entry()), 1)
    many = table(*[entry() for _ in range(300)])
    assert 100 * one < lib.puro_muon_direction_workspace_size(many, 300) < 140 * one
    shapes = table(*[entry(rows=64 + i) for i in range(20)])
    assert lib.puro_muon_direction_workspace_size(shapes, 20) < 12 * lib.puro_muon_direction_workspace_size(table(entry(rows=84)), 1)


def test_tables_are_checked():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        P.muon_table([(x, None, x)])  # not on CUDA


def test_struct_layout(tmp_path):
    """The Python mirror of puro_muon_matrix_t against the C compiler."""
    t = P.puro_muon_matrix_t
    fields = [f for f, _ in t._fields_]
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "puro_fp8.h"\nint main(void) { printf("%zu", sizeof(puro_muon_matrix_t));\n' +
                   "".join('printf(" %%zu", offsetof(puro_muon_matrix_t, %s));\n' % f for f in fields) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.dirname(P.HEADER_PATH), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(t)] + [getattr(t, f).offset for f in fields]
