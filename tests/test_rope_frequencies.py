"""Frequencies of the position rotation on the host, and what its entry points refuse (no GPU)."""
import ctypes
import math

import pytest
import torch

import _rope as R
import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import _build

BAD = P.PURO_ERR_INVALID_ARG
A = 0x100000  # an aligned address that nothing reads
KINDS = {"none": P.ROPE_NONE, "linear": P.ROPE_LINEAR, "base": P.ROPE_BASE, "turns": P.ROPE_TURNS, "index": P.ROPE_INDEX}


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return P.load_library()


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("rot,base,factor,trained", [(16, 1e4, 2.0, 4096), (128, 1e6, 4.0, 32768), (256, 5e5, 1.0, 8192), (64, 1e4, 32.0, 2048)])
def test_frequencies_are_the_definitions(lib, kind, rot, base, factor, trained):
    got = P.rope_frequencies(rot, base, KINDS[kind], factor, trained, 32.0, 1.0, device="cpu")
    want = R.frequencies(rot, base, kind, factor, trained, 32.0, 1.0)
    assert got.dtype == torch.int64 and got.shape == (rot // 2,)
    for g, w in zip(got.tolist(), want):
        # pow's argument and result, and the arithmetic of the ramp: ln(w) <= 16 times 2^-53, and a few times 2^-53
        assert abs((g % 2 ** 64) / 2 ** 64 - w / (2 * math.pi)) <= 2 ** -47 * w / (2 * math.pi) + 2 ** -64


def test_the_ramps_keep_fast_pairs_and_slow_slow_ones(lib):
    plain = P.rope_frequencies(128, 1e6, device="cpu")
    for kind in (P.ROPE_TURNS, P.ROPE_INDEX):
        f = P.rope_frequencies(128, 1e6, kind, 8.0, 32768, device="cpu")
        assert f[0] == plain[0] and abs(int(f[-1]) * 8 - int(plain[-1])) <= 16
        assert (f[1:] < f[:-1]).all()


def test_frequencies_refuse(lib):
    out = (ctypes.c_uint64 * 128)()
    good = [128, 1e6, P.ROPE_INDEX, 4.0, 32768, 32.0, 1.0, out]
    assert lib.puro_rope_frequencies(*good) == P.PURO_OK
    nan, inf = float("nan"), float("inf")
    for i, bads in ((0, (0, 8, 24, 272, -16)), (1, (1.0, 0.5, -2.0, nan, inf)), (2, (-1, 5)), (3, (0.5, nan, inf, -4.0)), (4, (0, -1)),
                    (5, (1.0, 0.5, nan, inf)), (6, (0.0, -1.0, 32.0, nan)), (7, (None,))):
        for bad in bads:
            args = list(good)
            args[i] = bad
            assert lib.puro_rope_frequencies(*args) == BAD, (i, bad)
    assert lib.puro_rope_frequencies(128, 1e300, P.ROPE_BASE, 1e10, 0, 0.0, 0.0, out) == BAD  # the base overflows
    assert lib.puro_rope_frequencies(128, 1e4, P.ROPE_NONE, nan, 0, nan, nan, out) == P.PURO_OK  # nothing of it is read
    with pytest.raises(ValueError):
        P.puro_rope_frequencies(128, 1e6, P.ROPE_NONE, 1.0, 0, 32.0, 1.0, torch.empty(63, dtype=torch.int64))
    with pytest.raises(P.PuroError):
        P.rope_frequencies(120, 1e6, device="cpu")


def test_tables_refuse(lib):
    good = [A, 128, 1.0, 5, 7, A, A, None]
    for i, bads in ((0, (None, A + 8)), (1, (0, 8, 40, 272)), (3, (-1, 2 ** 31 - 6)), (4, (-1, 2 ** 31 - 4)), (5, (None, A + 4)),
                    (6, (None, A + 8))):
        for bad in bads:
            args = list(good)
            args[i] = bad
            assert lib.puro_rope_tables(*args) == BAD, (i, bad)
    assert lib.puro_rope_tables(A, 128, 1.0, 0, 0, None, None, None) == P.PURO_OK


@pytest.mark.parametrize("name", ["puro_rope", "puro_rope_backward"])
def test_the_rotation_refuses(lib, name):
    fn = getattr(lib, name)

    def heads(n=4, data=A, ts=512, hs=128, reserved=0):
        return ctypes.byref(P.puro_heads_t(data, ts, hs, n, reserved))

    good = [heads(), heads(2), 5, 128, A, 128, 1.0, 0, A, heads(), heads(2), None]
    for i, bads in ((0, (heads(data=None), heads(data=A + 8), heads(ts=-8), heads(hs=4), heads(3), heads(reserved=1))),
                    (1, (heads(2, ts=7), heads(1), heads(-1))), (2, (-1,)), (3, (8, 120, 272, 64)), (4, (None, A + 8)),
                    (5, (0, 8, 24, 144, -16)), (8, (A + 2,)), (9, (heads(hs=64), heads(ts=64), heads(data=None), heads(3), None)),
                    (10, (heads(2, hs=120), heads(3)))):
        for bad in bads:
            args = list(good)
            args[i] = bad
            assert fn(*args) == BAD, (i, bad)
    for args in ([heads(0), heads(0), 5, 128, A, 128, 1.0, 0, A, heads(0), heads(0), None],
                 [None, None, 5, 128, A, 128, 1.0, 0, None, None, None, None],
                 [heads(data=None), heads(2, data=None), 0, 128, A, 128, 1.0, 0, A, heads(data=None), heads(2, data=None), None]):
        assert fn(*args) == P.PURO_OK  # nothing to do
    args = list(good)
    args[2] = 2 ** 31
    assert fn(*args) == P.PURO_ERR_UNSUPPORTED
