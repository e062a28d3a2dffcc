"""Backward of bias and activation, and of the gate, in BF16 and as FP8 copies, against 64 bits (_layer_ops.py)."""
import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P
from _parity import check_block_act_quant

DEV, BF, D64 = "cuda", torch.bfloat16, torch.float64
A = 0x100000
CODE = dict(zip(L.ACTS, (P.ACT_NONE, P.ACT_RELU, P.ACT_SILU, P.ACT_GELU, P.ACT_GELU_TANH)))
u8, f32 = torch.uint8, torch.float32


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _inputs(rows, cols, seed, n=2):
    """Values of all sizes that an activation meets: rows scaled by powers of two, zeros, far tails."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i in range(n):
        x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-4, 4, (rows, 1), generator=g))
        if i == 0:
            flat = x.view(-1)
            at = torch.randint(0, flat.numel(), (min(64, flat.numel()),), generator=g)
            flat[at] = torch.tensor([0.0, 40.0, -40.0, 90.0, -90.0, 300.0, -300.0, -0.0]).repeat(8)[:len(at)]
        out.append(x.to(BF))
    return out


def _quantized(rows, cols):
    op = lambda r, c: P.FP8Operand(torch.full((r, c), 0x55, dtype=u8, device=DEV),  # noqa: E731
                                   P.empty_scales(r, c, P.SCALE_BLOCK, P.ROLE_ACT, DEV).fill_(0x55))
    return P.Quantized(op(rows, cols), op(cols, rows))


def _copies(q):
    return q.rowwise.data, q.rowwise.scale, q.colwise.data, q.colwise.scale


def _close(got, ref, size):
    """Half a BF16 step and the FP32 error: a slope (of at most 1.2) is at most 2^-18 off -- 2^-22 of the exponential, as
    much of its argument's rounding times t |log t|, 2^-23 of the reciprocal, the products' roundings, times the inner
    slope of up to 3 where gelu_tanh's bell has not vanished --, an activation as much of max(1, |z|)."""
    assert bool(((got.cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18 * size).all())


def _close_sum(got, dz, dy):
    """The terms' errors, and a sum of at most rows / 8 + 64 roundings."""
    depth = dz.shape[0] / 8 + 64
    err = (got.cpu().double() - dz.sum(0)).abs()
    assert bool((err <= (2.0 ** -18 * dy.abs() + depth * 2.0 ** -24 * dz.abs()).sum(0) + 1e-30).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 40), (33, 256), (777, 264), (1337, 1536), (40000, 24)])
def test_bf16_form(rows, cols, act):
    _need_gpu()
    z, dy = _inputs(rows, cols, rows + cols)
    ref = dy.double() * L.slope(z.double(), act)
    zg, dyg = z.to(DEV), dy.to(DEV)
    dz, db = torch.full_like(dyg, 7.0), torch.full((cols,), 7.0, device=DEV)
    ws = torch.full((P.puro_act_backward_workspace_size(rows, cols),), 255, dtype=u8, device=DEV)
    P.puro_act_backward_bf16(dyg, None if act == "none" else zg, CODE[act], dz, db, ws)
    _close(dz, ref, dy.double().abs())
    _close_sum(db, ref, dy.double())
    only, inside = torch.zeros_like(db), dyg.clone()
    P.puro_act_backward_bf16(dyg, zg, CODE[act], None, only, ws)
    P.puro_act_backward_bf16(inside, zg, CODE[act], inside, None)
    assert torch.equal(only, db) and torch.equal(inside, dz)


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("rows,cols,fmt", [(128, 128, P.E4M3), (256, 640, P.E5M2), (1152, 1536, P.E4M3), (128, 8960, P.E4M3),
                                           (8192, 256, P.E4M3)])
def test_fp8_form(rows, cols, fmt, act):
    _need_gpu()
    z, dy = _inputs(rows, cols, rows + 3 * cols)
    ref = dy.double() * L.slope(z.double(), act)
    zg, dyg = None if act == "none" else z.to(DEV), dy.to(DEV)
    dz, db = torch.full_like(dyg, 7.0), torch.full((cols,), 7.0, device=DEV)
    ws = torch.full((P.puro_act_backward_workspace_size(rows, cols),), 255, dtype=u8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    q, q2, q3 = (_quantized(rows, cols) for _ in range(3))
    P.puro_fp8_quantize_act_backward(dyg, zg, CODE[act], fmt, dz, db, ws, *_copies(q), st)
    _close(dz, ref, dy.double().abs())
    _close_sum(db, ref, dy.double())
    check_block_act_quant(dz, q, fmt)
    db2 = torch.zeros_like(db)
    P.puro_fp8_quantize_act_backward(dyg, zg, CODE[act], fmt, None, db2, ws, *_copies(q2), st)
    P.puro_fp8_quantize_act_backward(dyg, zg, CODE[act], fmt, None, None, None, q3.rowwise.data, q3.rowwise.scale)
    assert torch.equal(db, db2) and all(torch.equal(a, b) for a, b in zip(_copies(q), _copies(q2)))
    assert all(torch.equal(a, b) for a, b in zip(_copies(q)[:2], _copies(q3)[:2])) and bool((q3.colwise.data == 0x55).all())
    assert int(st) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
def test_every_finite_value_through_the_slope(act):
    """dz of dy = 1, and [dgate, dup] of dh = up = 1: the slope, and the activation."""
    _need_gpu()
    z = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(BF)
    z = z[torch.isfinite(z)].view(-1, 8)
    one, dz = torch.ones_like(z), torch.empty_like(z)
    P.puro_act_backward_bf16(one, None if act == "none" else z, CODE[act], dz, None)
    zd = z.double().cpu()
    _close(dz, L.slope(zd, act), torch.ones_like(zd))
    out = torch.empty(z.shape[0], 16, dtype=BF, device=DEV)
    P.puro_gated_backward_bf16(one, z, one, CODE[act], out)
    _close(out[:, :8], L.slope(zd, act), torch.ones_like(zd))
    _close(out[:, 8:], L.act(zd, act), zd.abs().clamp(min=1))


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS[1:])
def test_far_and_not_finite_values(act):
    """Slopes at the ends: 0 and 1, NaN for NaN alone."""
    _need_gpu()
    big = float(torch.finfo(BF).max)
    z = torch.tensor([[big, -big, 1e30, -1e30, float("inf"), float("-inf"), float("nan"), -0.0]]).to(BF).to(DEV)
    dy = torch.full_like(z, 0.5)
    dz = torch.empty_like(z)
    P.puro_act_backward_bf16(dy, z, CODE[act], dz, None)
    half = 0.0 if act == "relu" else 0.25
    assert dz[0, :6].tolist() == [0.5, 0.0, 0.5, 0.0, 0.5, 0.0] and bool(torch.isnan(dz[0, 6])) and float(dz[0, 7]) == half


@pytest.mark.gpu
def test_not_finite_gradients_stay_in_their_groups():
    _need_gpu()
    z, dy = _inputs(256, 256, 5)
    dy[3, 7], dy[200, 130] = float("nan"), float("inf")
    q, dz = _quantized(256, 256), torch.empty(256, 256, dtype=BF, device=DEV)
    P.puro_fp8_quantize_act_backward(dy.to(DEV), z.to(DEV), P.ACT_SILU, P.E4M3, dz, None, None, *_copies(q))
    check_block_act_quant(dz, q, P.E4M3)
    assert int((~torch.isfinite(dz)).sum()) == 2


@pytest.mark.gpu
def test_no_rows_leave_a_zero_sum():
    _need_gpu()
    db = torch.full((8,), 3.0, device=DEV)
    P.puro_act_backward_bf16(torch.empty(0, 8, dtype=BF, device=DEV), None, P.ACT_NONE, None, db)
    assert bool((db == 0).all())


def _gates(rows, cols, seed):
    g, u, dh = _inputs(rows, cols, seed, 3)
    gu = torch.cat([g, u], 1).to(DEV)
    return g, u, dh, gu[:, :cols], gu[:, cols:], dh.to(DEV)


def _close_gated(got, dh, g, u, act):
    dg, du = L.gated_backward(dh.double(), g.double(), u.double(), act)
    c = dh.shape[1]
    _close(got[:, :c], dg, (dh.double() * u.double()).abs())
    _close(got[:, c:], du, dh.double().abs() * g.double().abs().clamp(min=1))


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 8), (5, 40), (130, 1544), (777, 256)])
def test_gated_bf16_form(rows, cols, act):
    _need_gpu()
    g, u, dh, gate, up, dhg = _gates(rows, cols, rows + cols)
    out = torch.full((rows, 2 * cols), 7.0, dtype=BF, device=DEV)
    P.puro_gated_backward_bf16(dhg, gate, up, CODE[act], out)
    _close_gated(out, dh, g, u, act)
    again = torch.empty_like(out)
    P.puro_gated_backward_bf16(dhg, gate.contiguous(), up.contiguous(), CODE[act], again)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("rows,cols,fmt", [(128, 128, P.E4M3), (256, 640, P.E5M2), (1152, 1536, P.E4M3), (128, 8960, P.E4M3)])
def test_gated_fp8_form(rows, cols, fmt, act):
    _need_gpu()
    g, u, dh, gate, up, dhg = _gates(rows, cols, rows + 5 * cols)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    q, q2, q3 = (_quantized(rows, 2 * cols) for _ in range(3))
    out = torch.full((rows, 2 * cols), 7.0, dtype=BF, device=DEV)
    P.puro_fp8_quantize_gated_backward(dhg, gate, up, CODE[act], fmt, out, *_copies(q), st)
    _close_gated(out, dh, g, u, act)
    check_block_act_quant(out, q, fmt)
    P.puro_fp8_quantize_gated_backward(dhg, gate, up, CODE[act], fmt, None, *_copies(q2), st)
    P.puro_fp8_quantize_gated_backward(dhg, gate, up, CODE[act], fmt, None, q3.rowwise.data, q3.rowwise.scale)
    assert all(torch.equal(a, b) for a, b in zip(_copies(q), _copies(q2)))
    assert all(torch.equal(a, b) for a, b in zip(_copies(q)[:2], _copies(q3)[:2]))
    both = torch.empty_like(out)
    P.puro_gated_backward_bf16(dhg, gate, up, CODE[act], both)
    assert torch.equal(both, out) and int(st) == 0


@pytest.mark.gpu
def test_gated_not_finite_values_stay_in_their_groups():
    _need_gpu()
    g, u, dh, gate, up, dhg = _gates(128, 256, 9)
    dhg[1, 200], gate[77, 3] = float("inf"), float("nan")
    q, out = _quantized(128, 512), torch.empty(128, 512, dtype=BF, device=DEV)
    P.puro_fp8_quantize_gated_backward(dhg, gate, up, P.ACT_SILU, P.E4M3, out, *_copies(q))
    check_block_act_quant(out, q, P.E4M3)


# ------------------------------------------------------------- refusals, without a GPU
def test_act_backward_refusals():
    lib, bad = P.load_library(), P.PURO_ERR_INVALID_ARG
    size = P.puro_act_backward_workspace_size

    def bf16(dy=A, z=A, r=3, c=16, act=2, dz=A, db=A, ws=A, n=1 << 30):
        return lib.puro_act_backward_bf16(dy, z, r, c, act, dz, db, ws, n, None)

    def fp8(dy=A, z=A, r=128, c=256, act=2, fmt=0, dz=A, db=A, ws=A, n=1 << 30, q=A, s=A, qt=A, stt=A):
        return lib.puro_fp8_quantize_act_backward(dy, z, r, c, act, fmt, dz, db, ws, n, q, s, qt, stt, None, None)

    for kw in (dict(act=5), dict(act=-1), dict(r=-1), dict(dy=None), dict(z=None), dict(dy=A + 2), dict(z=A + 8), dict(dz=A + 8),
               dict(db=A + 2), dict(ws=None), dict(ws=A + 4)):
        assert bf16(**kw) == bad and fp8(**kw) == bad, kw
    assert bf16(c=12) == bad and bf16(n=size(3, 16) - 1) == bad
    for kw in (dict(r=130), dict(c=200), dict(fmt=2), dict(q=None), dict(s=None), dict(q=A + 8), dict(qt=None), dict(stt=None),
               dict(stt=A + 8), dict(n=size(128, 256) - 1)):
        assert fp8(**kw) == bad, kw
    assert bf16(r=2 ** 31) == P.PURO_ERR_UNSUPPORTED
    assert bf16(r=0, db=None) == fp8(r=0, db=None) == bf16(c=0) == bf16(dz=None, db=None) == P.PURO_OK
    assert bf16(z=None, act=0, dz=None, db=None) == P.PURO_OK


def test_act_backward_workspace():
    size = P.puro_act_backward_workspace_size
    for r, c in ((1, 8), (128, 8960), (8192, 128), (1337, 1536), (10 ** 6, 64)):
        n = size(r, c)
        assert n % (4 * c) == 0 and n >= 4 * c * -(-r // 128) and n <= 4 * c * -(-r // 32)
    assert size(0, 8) == size(8, 0) == 0


def test_gated_backward_refusals():
    lib, bad = P.load_library(), P.PURO_ERR_INVALID_ARG

    def bf16(dh=A, g=A, u=A, r=3, c=16, ld=32, act=2, out=A):
        return lib.puro_gated_backward_bf16(dh, g, u, r, c, ld, act, out, None)

    def fp8(dh=A, g=A, u=A, r=128, c=256, ld=512, act=2, fmt=0, out=A, q=A, s=A, qt=A, stt=A):
        return lib.puro_fp8_quantize_gated_backward(dh, g, u, r, c, ld, act, fmt, out, q, s, qt, stt, None, None)

    for kw in (dict(act=5), dict(act=-1), dict(r=-1), dict(dh=None), dict(g=None), dict(u=None), dict(dh=A + 2), dict(g=A + 8),
               dict(u=A + 4), dict(out=A + 8), dict(ld=8), dict(ld=513)):
        assert bf16(**kw) == bad and fp8(**kw) == bad, kw
    assert bf16(c=12) == bad and bf16(out=None) == bad
    for kw in (dict(r=130), dict(c=200), dict(fmt=2), dict(q=None), dict(s=None), dict(qt=None), dict(stt=None), dict(qt=A + 8)):
        assert fp8(**kw) == bad, kw
    assert fp8(c=2 ** 30, ld=2 ** 30) == P.PURO_ERR_UNSUPPORTED
    assert bf16(r=0) == fp8(r=0) == P.PURO_OK
