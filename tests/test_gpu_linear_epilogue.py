"""Linears with bias, activation and residual in the epilogue, and the gated
MLP's two projections in one kernel, against 64 bits (_layer_ops.py)."""
import ctypes

import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P
from _parity import check_block_act_quant, scales_of

DEV, BF, D64, u8 = "cuda", torch.bfloat16, torch.float64, torch.uint8
A = 0x100000
CODE = dict(zip(L.ACTS, (P.ACT_NONE, P.ACT_RELU, P.ACT_SILU, P.ACT_GELU, P.ACT_GELU_TANH)))
F8 = {P.E4M3: torch.float8_e4m3fn, P.E5M2: torch.float8_e5m2}


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _normal(shape, std, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(BF)


def _operand(v, ops, role):
    """The operand the call takes and its values in 64 bits."""
    if ops == "bf16":
        return v, v.double()
    sc = P.SCALE_BLOCK if ops == "block" else P.SCALE_TENSOR
    q = P.quantize(v, P.E4M3, sc, role, transpose=False).rowwise
    codes = q.data.view(F8[P.E4M3]).double()
    if ops == "tensor":
        return q, codes * q.scale.double()
    s = torch.from_numpy(scales_of(q)).to(DEV).double()
    return q, codes * torch.exp2(s - 127).repeat_interleave(128, 1)


def _product(x, w, ops):
    """x w^T in 64 bits and what an FP32 accumulation may be off by: a chain of at most K / 16 + 64 additions, each at most
    2^-23 of the sum of magnitudes."""
    return x @ w.t(), (x.shape[1] / 16 + 64) * 2.0 ** -23 * (x.abs() @ w.abs().t())


def _act_error(z, err):
    """An activation's error in FP32 (2^-18 of max(1, |z|), test_gpu_act_backward.py) behind an argument off by err (slopes
    are below 1.2)."""
    return 1.2 * err + 2.0 ** -18 * z.abs().clamp(min=1)


def _within(got, ref, err):
    """Half a BF16 step (2^-8 of the value) and the error before the rounding."""
    bad = (got.double() - ref).abs() > 2.0 ** -8 * (ref.abs() + err) + err
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}"


def _workspace(ops, m, n, k, give):
    size = P.puro_fp8_workspace_size(m, n, k) if ops != "bf16" and give else 0
    return torch.full((size,), 255, dtype=u8, device=DEV) if size else None


def _linear(ops, x, w, y, bias=None, act="none", residual=None, z=None, ws=None, st=None, stream=None):
    if ops == "bf16":
        P.puro_bf16_linear_fprop_epilogue(x, w, y, bias, CODE[act], residual, z, st, stream)
    else:
        P.puro_fp8_linear_fprop_epilogue(x, w, y, bias, CODE[act], residual, z, ws, st, stream)


SHAPES = [("block", 128, 128, 128, False), ("block", 256, 384, 512, False), ("block", 384, 1536, 1536, False),
          ("block", 256, 1536, 8960, True), ("block", 128, 256, 4096, True), ("block", 2048, 1536, 8960, True),
          ("block", 1152, 2048, 2048, False), ("block", 8192, 2048, 256, False), ("tensor", 16, 48, 32, False),
          ("tensor", 272, 1552, 208, False), ("tensor", 256, 1536, 4096, True), ("tensor", 128, 256, 2048, True),
          ("bf16", 1, 8, 8, False), ("bf16", 3, 40, 72, False), ("bf16", 17, 264, 136, False), ("bf16", 77, 1544, 520, False),
          ("bf16", 300, 2048, 1536, False), ("bf16", 1, 1536, 8960, False), ("bf16", 8, 1544, 2000, False),
          ("bf16", 16, 1536, 1544, False), ("bf16", 33, 1536, 1536, False), ("bf16", 64, 8960, 1536, False),
          ("bf16", 130, 136, 4096, False), ("bf16", 1000, 512, 64, False), ("bf16", 513, 1800, 256, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("ops,m,n,k,give", SHAPES)
def test_linear(ops, m, n, k, give):
    _need_gpu()
    (x, xd), (w, wd) = _operand(_normal((m, k), 1.0, 1), ops, P.ROLE_ACT), _operand(_normal((n, k), 0.03, 2), ops, P.ROLE_WEIGHT)
    bias, wide = _normal((n,), 0.5, 3), _normal((m, n + 24), 1.0, 4)
    residual = wide[:, 8:n + 8]
    prod, err = _product(xd, wd, ops)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for act, b, r, keep in (("none", None, residual, False), ("gelu", bias, residual, True), ("silu", bias, None, False),
                            ("relu", None, None, True), ("gelu_tanh", bias, residual.contiguous(), True), ("none", bias, None, True),
                            ("none", None, None, False)):
        y = torch.full((m + 2, n), 7.0, dtype=BF, device=DEV)
        z = torch.full((m + 2, n), 7.0, dtype=BF, device=DEV) if keep else None
        _linear(ops, x, w, y[1:-1], b, act, r, None if z is None else z[1:-1], _workspace(ops, m, n, k, give), st)
        zr = prod if b is None else prod + b.double()
        e = err + (0 if b is None else 2.0 ** -23 * (zr.abs() + err))
        yr = L.act(zr, act)
        ye = e if act == "none" else _act_error(zr, e)
        if r is not None:
            yr = yr + r.double()
            ye = ye + 2.0 ** -23 * (yr.abs() + ye)
        _within(y[1:-1], yr, ye)
        assert bool((y[0] == 7).all() and (y[-1] == 7).all())
        if keep:
            _within(z[1:-1], zr, e)
            assert bool((z[0] == 7).all() and (z[-1] == 7).all())
    assert int(st) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("ops,m,n,k,give", [("block", 256, 1536, 1536, False), ("block", 256, 1536, 8960, True),
                                            ("block", 2048, 1536, 8960, True), ("bf16", 333, 1536, 512, False),
                                            ("bf16", 5, 1536, 512, False)])
def test_residual_in_place_streams_and_graphs(ops, m, n, k, give):
    """y = y + x w^T, on another stream, captured and replayed: the same bytes."""
    _need_gpu()
    x, w = (_operand(v, ops, r)[0] for v, r in ((_normal((m, k), 1.0, 5), P.ROLE_ACT), (_normal((n, k), 0.03, 6), P.ROLE_WEIGHT)))
    start = _normal((m, n), 1.0, 7)
    want, ws = torch.empty_like(start), _workspace(ops, m, n, k, give)
    _linear(ops, x, w, want, residual=start, ws=ws)
    y = start.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _linear(ops, x, w, y, residual=y, ws=ws, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _linear(ops, x, w, y, residual=y, ws=ws)
    for _ in range(2):
        y.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.gpu
def test_empty_extents():
    _need_gpu()
    bias, res = _normal((16,), 1.0, 1), _normal((3, 16), 1.0, 2)
    e = lambda *s: torch.empty(s, dtype=BF, device=DEV)  # noqa: E731
    y, z = e(3, 16), e(3, 16)
    P.puro_bf16_linear_fprop_epilogue(e(3, 0), e(16, 0), y, bias, P.ACT_SILU, res, z)
    assert torch.equal(z, bias.expand(3, 16))
    _within(y, L.act(bias.double(), "silu") + res.double(), 2.0 ** -17 * torch.ones(3, 16, dtype=D64, device=DEV) * 4)
    P.puro_bf16_linear_fprop_epilogue(e(0, 8), e(16, 8), e(0, 16), bias)
    h, gu = torch.full((3, 8), 7.0, dtype=BF, device=DEV), torch.full((3, 16), 7.0, dtype=BF, device=DEV)
    P.puro_bf16_gated_fprop(e(3, 0), e(16, 0), P.ACT_SILU, gu, h)
    assert bool((h == 0).all() and (gu == 0).all())


@pytest.mark.gpu
def test_not_finite_values_stay_in_their_rows():
    _need_gpu()
    x, w = _normal((40, 256), 1.0, 1), _normal((136, 256), 0.05, 2)
    x[7, 3], x[20, 100] = float("nan"), float("inf")
    y = torch.empty(40, 136, dtype=BF, device=DEV)
    P.puro_bf16_linear_fprop_epilogue(x, w, y)
    bad = ~torch.isfinite(y).all(1)
    assert bad.nonzero().flatten().tolist() == [7, 20]


@pytest.mark.gpu
@pytest.mark.parametrize("m", [8160, 16])
@pytest.mark.parametrize("act", L.ACTS)
def test_every_finite_value_through_the_activation(act, m):
    """x times the identity is x, exactly, so y is the activation of every finite BF16 value."""
    _need_gpu()
    x = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(BF)
    x = x[torch.isfinite(x)].view(m, -1)
    eye = torch.eye(x.shape[1], dtype=BF, device=DEV)
    y, h = torch.empty_like(x), torch.empty_like(x)
    P.puro_bf16_linear_fprop_epilogue(x, eye, y, None, CODE[act])
    ref, err = L.act(x.double(), act), 0 if act in ("none", "relu") else _act_error(x.double(), 0)
    _within(y, ref, err + torch.zeros_like(ref))
    P.puro_bf16_gated_fprop(x, torch.cat([eye, eye]), CODE[act], None, h)
    small = x.double().abs() < 1e15  # (the product is finite)
    # (below 2^-126 half a BF16 step is 2^-134, whatever the value, and FP32's 2^-150)
    _within(h[small], (ref * x.double())[small], ((err + 2.0 ** -23 * ref.abs()) * x.double().abs())[small] + 2.0 ** -133)


def _quantized(rows, cols):
    op = lambda r, c: P.FP8Operand(torch.full((r, c), 0x55, dtype=u8, device=DEV),  # noqa: E731
                                   P.empty_scales(r, c, P.SCALE_BLOCK, P.ROLE_ACT, DEV).fill_(0x55))
    return P.Quantized(op(rows, cols), op(cols, rows))


def _copies(q):
    return q.rowwise.data, q.rowwise.scale, q.colwise.data, q.colwise.scale


def _check_gated(x, w, act, gate_up, h):
    f = w.shape[0] // 2
    prod, err = _product(x, w, None)
    g, u, ge, ue = prod[:, :f], prod[:, f:], err[:, :f], err[:, f:]
    if gate_up is not None:
        _within(gate_up, prod, err)
    a = L.act(g, act)
    ae = ge if act == "none" else _act_error(g, ge)
    he = ae * u.abs() + (a.abs() + ae) * ue
    _within(h, a * u, he + 2.0 ** -23 * (a * u).abs())


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("m,f,k,fmt", [(128, 128, 128, P.E4M3), (256, 640, 384, P.E5M2), (384, 1536, 1536, P.E4M3),
                                       (1152, 1280, 256, P.E4M3), (2048, 8960, 256, P.E4M3)])
def test_gated_fp8(m, f, k, fmt, act):
    _need_gpu()
    (x, xd), (w, wd) = _operand(_normal((m, k), 1.0, 1), "block", P.ROLE_ACT), _operand(_normal((2 * f, k), 0.05, 2), "block", P.ROLE_WEIGHT)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    q, q2, q3 = (_quantized(m, f) for _ in range(3))
    gu, h = (torch.full((m, c), 7.0, dtype=BF, device=DEV) for c in (2 * f, f))
    P.puro_fp8_gated_fprop(x, w, CODE[act], fmt, gu, h, *_copies(q), st)
    _check_gated(xd, wd, act, gu, h)
    check_block_act_quant(h, q, fmt)
    P.puro_fp8_gated_fprop(x, w, CODE[act], fmt, None, None, *_copies(q2), st)
    P.puro_fp8_gated_fprop(x, w, CODE[act], fmt, None, None, q3.rowwise.data, q3.rowwise.scale)
    assert all(torch.equal(a, b) for a, b in zip(_copies(q), _copies(q2)))
    assert all(torch.equal(a, b) for a, b in zip(_copies(q)[:2], _copies(q3)[:2])) and bool((q3.colwise.data == 0x55).all())
    assert int(st) == 0


@pytest.mark.gpu
def test_gated_fp8_not_finite_groups():
    _need_gpu()
    xv = _normal((256, 256), 1.0, 1)
    xv[5, 9], xv[200, 130] = float("nan"), float("inf")
    x, w = _operand(xv, "block", P.ROLE_ACT)[0], _operand(_normal((512, 256), 0.05, 2), "block", P.ROLE_WEIGHT)[0]
    q, h = _quantized(256, 256), torch.empty(256, 256, dtype=BF, device=DEV)
    P.puro_fp8_gated_fprop(x, w, P.ACT_SILU, P.E4M3, None, h, *_copies(q))
    check_block_act_quant(h, q, P.E4M3)
    assert (~torch.isfinite(h).all(1)).nonzero().flatten().tolist() == [5, 200]


@pytest.mark.gpu
def test_gated_fp8_empty_reduction():
    _need_gpu()
    e = lambda r, c: torch.empty((r, c), dtype=u8, device=DEV)  # noqa: E731
    some = torch.zeros(512, dtype=u8, device=DEV)
    q = _quantized(128, 256)
    r = ctypes.byref
    x = P.puro_fp8_tensor_t(some.data_ptr(), some.data_ptr(), 128, 0, 0, 1, 0, 0)
    w = P.puro_fp8_tensor_t(some.data_ptr(), some.data_ptr(), 512, 0, 0, 1, 1, 0)
    gu = torch.full((128, 512), 7.0, dtype=BF, device=DEV)
    assert P.load_library().puro_fp8_gated_fprop(r(x), r(w), P.ACT_SILU, 0, gu.data_ptr(), None, *[t.data_ptr() for t in _copies(q)],
                                                 None, torch.cuda.current_stream().cuda_stream) == P.PURO_OK
    check_block_act_quant(torch.zeros(128, 256, dtype=BF, device=DEV), q, P.E4M3)
    assert bool((gu == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("m,f,k", [(1, 8, 8), (5, 40, 72), (77, 136, 520), (300, 1000, 264), (1, 8960, 1536), (600, 896, 128),
                                   (16, 1544, 1000), (40, 2048, 264)])
def test_gated_bf16(m, f, k, act):
    _need_gpu()
    x, w = _normal((m, k), 1.0, 1), _normal((2 * f, k), 0.05, 2)
    h, gu = (torch.full((m + 2, c), 7.0, dtype=BF, device=DEV) for c in (f, 2 * f))
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.puro_bf16_gated_fprop(x, w, CODE[act], gu[1:-1], h[1:-1], st)
    _check_gated(x.double(), w.double(), act, gu[1:-1], h[1:-1])
    assert all(bool((t[i] == 7).all()) for t in (h, gu) for i in (0, -1))
    only = torch.empty(m, f, dtype=BF, device=DEV)
    P.puro_bf16_gated_fprop(x, w, CODE[act], None, only)
    assert torch.equal(only, h[1:-1]) and int(st) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["linear_block", "linear_tensor", "linear_bf16", "gated_bf16", "gated_block"])
def test_a_wait_that_runs_out_is_reported(kind):
    """As in test_gpu_faults.py: a zero bound on every wait, then the same call again."""
    _need_gpu()
    m, n, k = 4096, 2048, 4096
    ops = kind.split("_")[1]
    (x, xd), (w, wd) = _operand(_normal((m, k), 1.0, 3), ops, P.ROLE_ACT), _operand(_normal((n, k), 0.02, 4), ops, P.ROLE_WEIGHT)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    y, h, q = (torch.empty(m, c, dtype=BF, device=DEV) for c in (n, n // 2, 8))
    q = _quantized(m, n // 2)
    if kind == "gated_bf16":
        run = lambda: P.puro_bf16_gated_fprop(x, w, P.ACT_SILU, None, h, st)  # noqa: E731
    elif kind == "gated_block":
        run = lambda: P.puro_fp8_gated_fprop(x, w, P.ACT_SILU, P.E4M3, None, h, *_copies(q), st)  # noqa: E731
    else:
        run = lambda: _linear(ops, x, w, y, act="silu", st=st)  # noqa: E731
    torch.cuda.synchronize()
    P.puro_set_wait_timeout_ns(0)
    try:
        run()
        torch.cuda.synchronize()
    finally:
        P.puro_set_wait_timeout_ns(2_000_000_000)
    assert P.puro_fp8_get_status(st) == P.PURO_ERR_TIMEOUT
    st.zero_()
    run()
    assert P.puro_fp8_get_status(st) == P.PURO_OK
    if kind.startswith("gated"):
        _check_gated(xd, wd, "silu", None, h)
        if kind == "gated_block":
            check_block_act_quant(h, q, P.E4M3)
    else:
        z, err = _product(xd, wd, ops)
        _within(y, L.act(z, "silu"), _act_error(z, err))


# ------------------------------------------------------------- refusals, without a GPU
def _op(rows, red, scaling=P.SCALE_BLOCK, role=P.ROLE_ACT, data=A):
    return P.puro_fp8_tensor_t(data, A, rows, red, 0, scaling, role, 0)


def test_linear_refusals():
    lib, bad, r = P.load_library(), P.PURO_ERR_INVALID_ARG, ctypes.byref

    def fp8(x=_op(256, 384), w=_op(512, 384, role=1), bias=A, act=0, res=A, ld=512, z=A, y=A):
        return lib.puro_fp8_linear_fprop_epilogue(r(x), r(w), bias, act, res, ld, z, y, None, 0, None, None)

    def bf16(x=A, w=A, m=3, n=16, k=8, bias=A, act=0, res=A, ld=16, z=A, y=A):
        return lib.puro_bf16_linear_fprop_epilogue(x, w, m, n, k, bias, act, res, ld, z, y, None, None)

    for kw in (dict(bias=A + 2), dict(act=5), dict(act=-1), dict(res=A + 8), dict(ld=8), dict(ld=516), dict(z=A + 2), dict(y=None),
               dict(y=A + 4)):
        assert fp8(**kw) == bad and bf16(**kw) == bad, kw
    for kw in (dict(x=_op(256, 256)), dict(x=_op(200, 384)), dict(w=_op(512, 384, P.SCALE_TENSOR)), dict(x=_op(256, 384, data=None))):
        assert fp8(**kw) == bad, kw
    for kw in (dict(m=-1), dict(n=12, ld=16), dict(k=12), dict(x=None), dict(w=None), dict(x=A + 8), dict(w=A + 2)):
        assert bf16(**kw) == bad, kw
    assert bf16(m=2 ** 31) == P.PURO_ERR_UNSUPPORTED
    assert bf16(m=0, y=None) == bf16(n=0) == P.PURO_OK and fp8(x=_op(0, 384)) == P.PURO_OK


def test_gated_refusals():
    lib, bad, r = P.load_library(), P.PURO_ERR_INVALID_ARG, ctypes.byref

    def fp8(x=_op(256, 384), w=_op(512, 384, role=1), act=2, fmt=0, gu=A, h=A, q=A, s=A, qt=A, stt=A):
        return lib.puro_fp8_gated_fprop(r(x), r(w), act, fmt, gu, h, q, s, qt, stt, None, None)

    def bf16(x=A, w=A, m=3, f=16, k=8, act=2, gu=A, h=A):
        return lib.puro_bf16_gated_fprop(x, w, m, f, k, act, gu, h, None, None)

    for kw in (dict(act=5), dict(act=-1), dict(gu=A + 2), dict(h=A + 8)):
        assert fp8(**kw) == bad and bf16(**kw) == bad, kw
    for kw in (dict(fmt=2), dict(q=None), dict(s=None), dict(qt=None), dict(stt=None), dict(q=A + 8), dict(w=_op(384, 384, role=1)),
               dict(w=_op(512, 256, role=1)), dict(x=_op(256, 384, P.SCALE_TENSOR))):
        assert fp8(**kw) == bad, kw
    for kw in (dict(m=-1), dict(f=12), dict(k=4), dict(x=None), dict(w=None), dict(h=None), dict(w=A + 2)):
        assert bf16(**kw) == bad, kw
    assert bf16(f=2 ** 30) == P.PURO_ERR_UNSUPPORTED
    assert bf16(m=0, h=None) == P.PURO_OK and fp8(x=_op(0, 384)) == P.PURO_OK
