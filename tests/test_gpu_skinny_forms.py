"""Linears and gated MLPs of a few tokens, against 64 bits, at widths that take each of the forms of csrc/skinny_plan.h
(16, 8, 12, 6 and 4 warps a block on 152 SMs, in this order) and at the widths beside 8960."""
import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P
import test_gpu_linear_epilogue as T

BF, DEV = torch.bfloat16, "cuda"


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 8, 13])
@pytest.mark.parametrize("n,k", [(512, 1544), (8960, 520), (4096, 2056), (7168, 2048), (9752, 4096), (9064, 264), (9072, 264), (9216, 264)])
def test_linear(n, k, m):
    _linear(m, n, k)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [17, 32])
@pytest.mark.parametrize("n,k", [(512, 1000), (4096, 1000), (8000, 384)])
def test_linear_of_small_weights(n, k, m):
    _linear(m, n, k)


def _linear(m, n, k):
    T._need_gpu()
    x, w, bias, res = T._normal((m, k), 1.0, 1), T._normal((n, k), 0.03, 2), T._normal((n,), 0.5, 3), T._normal((m, n), 1.0, 4)
    prod, err = T._product(x.double(), w.double(), "bf16")
    y, z = (torch.full((m + 2, n), 7.0, dtype=BF, device=DEV) for _ in range(2))
    P.puro_bf16_linear_fprop_epilogue(x, w, y[1:-1], bias, P.ACT_GELU, res, z[1:-1])
    zr = prod + bias.double()
    e = err + 2.0 ** -23 * (zr.abs() + err)
    yr = L.act(zr, "gelu") + res.double()
    ye = T._act_error(zr, e)
    T._within(z[1:-1], zr, e)
    T._within(y[1:-1], yr, ye + 2.0 ** -23 * (yr.abs() + ye))
    assert all(bool((t[i] == 7).all()) for t in (y, z) for i in (0, -1))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 8, 13])
@pytest.mark.parametrize("f,k", [(1024, 1000), (4096, 520), (3648, 2048), (6144, 520), (7344, 8960), (9216, 264)])
def test_gated(f, k, m):
    _gated(m, f, k)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [17, 32])
@pytest.mark.parametrize("f,k", [(1000, 520), (2048, 1000), (1240, 1536), (3704, 512), (5000, 256)])
def test_gated_of_small_weights(f, k, m):
    _gated(m, f, k)


def _gated(m, f, k):
    T._need_gpu()
    x, w = T._normal((m, k), 1.0, 1), T._normal((2 * f, k), 0.03, 2)
    h, gu = (torch.full((m + 2, c), 7.0, dtype=BF, device=DEV) for c in (f, 2 * f))
    P.puro_bf16_gated_fprop(x, w, P.ACT_SILU, gu[1:-1], h[1:-1])
    T._check_gated(x.double(), w.double(), "silu", gu[1:-1], h[1:-1])
    assert all(bool((t[i] == 7).all()) for t in (h, gu) for i in (0, -1))


@pytest.mark.gpu
def test_gated_bf16_several_tiles_a_pair():
    """The form that takes over from these: 187 tiles on 76 pairs of SMs, ragged both ways."""
    _gated(2600, 2056, 264)
