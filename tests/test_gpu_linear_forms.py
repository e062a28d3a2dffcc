"""The tile forms of linears with an epilogue, each by shapes that take it, against 64 bits: 256-wide tiles (the form of
large linears: registers split between the warps' roles, a one-kilobyte store ring) and 192-wide ones for each type of
operand, several tiles a pair of SMs, and a reduction split through memory with scales per tensor.

What form a shape takes is the cost model of csrc/gemm.cu, repeated here, so that a test whose shape no longer takes
its form says so; puro_set_gemm_tile_n(256) makes every tile 256 wide that is neither split nor shared by a cluster."""
import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P
import test_gpu_linear_epilogue as T

DEV, BF = "cuda", torch.bfloat16
PAIRS, COSTS = 76, ((256, 131, 900), (192, 120, 500), (128, 95, 400))


def _ceil(a, b):
    return -(-a // b)


def _tiles(m, n, width):
    return _ceil(m, 256) * _ceil(n, width)


def _cycles(cost, red):
    return _ceil(red, 128) * 4 * cost[1] + cost[2]


def _width(m, n, red):
    best, least = 256, 0
    for c in COSTS:
        cycles = _ceil(_tiles(m, n, c[0]), PAIRS) * _cycles(c, red)
        if c[0] == 256 or cycles * 100 < least * 97:
            best, least = c[0], cycles
    return best


def _form(ops, m, n, k, give):
    """The tile's width, "memory", or "shared" where clusters might share the reduction."""
    red = 2 * k if ops == "bf16" else k
    clusters = any(_tiles(m, n, 128) <= most and _ceil(red, 256) >= 2 * pairs for pairs, most in ((4, 15), (2, 36)))
    if ops == "bf16":
        assert m > 32  # (there is a form for a few tokens)
    elif not (give and P.puro_fp8_workspace_size(m, n, k)):
        clusters = False
    elif not clusters:
        return "memory"
    return "shared" if clusters else _width(m, n, red)


def _check(ops, m, n, k, give):
    (x, xd), (w, wd) = T._operand(T._normal((m, k), 1.0, 1), ops, P.ROLE_ACT), T._operand(T._normal((n, k), 0.03, 2), ops, P.ROLE_WEIGHT)
    bias, wide = T._normal((n,), 0.5, 3), T._normal((m, n + 24), 1.0, 4)
    narrow = wide[:, 8:n + 8]  # rows at 16 bytes
    whole = narrow.contiguous()
    prod, err = T._product(xd, wd, ops)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for act, b, r, keep, inside in (("none", None, narrow, False, False), ("gelu", bias, narrow, True, False),
                                    ("silu", bias, whole, False, True), ("relu", None, None, True, False),
                                    ("gelu_tanh", bias, whole, True, True), ("none", None, whole, False, True),
                                    ("none", bias, None, True, False)):
        y = torch.full((m + 2, n), 7.0, dtype=BF, device=DEV)
        z = torch.full((m + 2, n), 7.0, dtype=BF, device=DEV) if keep else None
        if inside:
            y[1:-1] = r
        T._linear(ops, x, w, y[1:-1], b, act, y[1:-1] if inside else r, None if z is None else z[1:-1],
                  T._workspace(ops, m, n, k, give), st)
        zr = prod if b is None else prod + b.double()
        e = err + (0 if b is None else 2.0 ** -23 * (zr.abs() + err))
        yr, ye = L.act(zr, act), e if act == "none" else T._act_error(zr, e)
        if r is not None:
            yr = yr + r.double()
            ye = ye + 2.0 ** -23 * (yr.abs() + ye)
        T._within(y[1:-1], yr, ye)
        assert bool((y[0] == 7).all() and (y[-1] == 7).all())
        if keep:
            T._within(z[1:-1], zr, e)
            assert bool((z[0] == 7).all() and (z[-1] == 7).all())
    assert int(st) == 0


@pytest.fixture
def all_256_wide():
    P.puro_set_gemm_tile_n(256)
    yield
    P.puro_set_gemm_tile_n(0)


# fewer tiles than pairs, more tiles than pairs; ragged rows and columns where the operands allow them (n * 2 bytes a
# multiple of 32 and not, so that rows leave and residuals come directly and through the staging)
@pytest.mark.gpu
@pytest.mark.parametrize("ops,m,n,k", [("block", 384, 640, 256), ("block", 4992, 1152, 384), ("tensor", 1808, 784, 48),
                                       ("tensor", 5008, 1296, 144), ("bf16", 1800, 776, 72), ("bf16", 5001, 1288, 136),
                                       ("bf16", 2600, 2064, 520)])
def test_256_wide_tiles(ops, m, n, k, all_256_wide):
    T._need_gpu()
    assert isinstance(_form(ops, m, n, k, False), int)
    _check(ops, m, n, k, False)


@pytest.mark.gpu
@pytest.mark.parametrize("ops,m,n,k", [("block", 5120, 2304, 1536), ("tensor", 5104, 2288, 1040), ("bf16", 5001, 2296, 520)])
def test_256_wide_tiles_by_the_model(ops, m, n, k):
    T._need_gpu()
    assert _form(ops, m, n, k, False) == 256
    _check(ops, m, n, k, False)


@pytest.mark.gpu
@pytest.mark.parametrize("ops,m,n,k", [("block", 1280, 2048, 256), ("block", 2304, 2560, 384), ("tensor", 1296, 1808, 144),
                                       ("tensor", 1808, 2576, 48), ("bf16", 1300, 1800, 264), ("bf16", 1801, 2568, 72)])
def test_192_wide_tiles(ops, m, n, k):
    T._need_gpu()
    assert _form(ops, m, n, k, False) == 192
    _check(ops, m, n, k, False)


@pytest.mark.gpu
@pytest.mark.parametrize("ops", ["tensor", "block"])
def test_reduction_split_through_memory(ops):
    """Scales per tensor are applied to each partial product, once, ahead of bias and activation."""
    T._need_gpu()
    assert _form(ops, 2048, 1536, 8960, True) == "memory"
    _check(ops, 2048, 1536, 8960, True)


def test_the_forms_of_the_shapes():
    """The same assertions without a GPU."""
    for ops, m, n, k, form in (("block", 5120, 2304, 1536, 256), ("tensor", 5104, 2288, 1040, 256), ("bf16", 5001, 2296, 520, 256),
                               ("block", 1280, 2048, 256, 192), ("bf16", 1801, 2568, 72, 192)):
        assert _form(ops, m, n, k, False) == form, (ops, m, n, k)
    assert _form("tensor", 2048, 1536, 8960, True) == "memory"
