"""Query and key norms with the position rotation, forward and backward,
against 64 bits (_layer_ops.py)."""
import ctypes

import pytest
import torch

import _layer_ops as L
import paper_2608_27370_gb300 as P

DEV, EPS, D64, BF = "cuda", 1e-6, torch.float64, torch.bfloat16
A = 0x100000  # an aligned address that nothing reads


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def tables(n, rot, base=1e4):
    a = torch.arange(n, dtype=D64)[:, None] * base ** (-2 * torch.arange(rot // 2, dtype=D64) / max(rot, 1))
    return a.cos().float(), a.sin().float()


class Case:
    """Inputs on the CPU and the GPU, and the 64-bit results."""

    def __init__(self, t, hq, hkv, d, rot, inter, positions="arange", gains=True, seed=0):
        g = torch.Generator().manual_seed(1000 * d + 10 * t + seed)
        r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.t, self.hq, self.hkv, self.d, self.rot, self.inter = t, hq, hkv, d, rot, inter
        self.qkv = (r(t, (hq + 2 * hkv) * d) * torch.exp2(torch.randint(-3, 4, (t, 1), generator=g))).to(BF)
        self.gains = [(1 + 0.3 * r(d)).to(BF) if gains else None for _ in range(2)]
        self.dy = [r(t, h, d).to(BF) for h in (hq, hkv)]
        n = t + 5
        self.cos, self.sin = tables(n, rot)
        self.positions = None
        if positions == "packed":  # two sequences and padding behind them
            used = t - t // 4
            self.positions = torch.cat([torch.arange(used // 2), torch.arange(used - used // 2), torch.full((t - used,), -1)]).int()
        elif positions == "shuffled":
            self.positions = torch.randperm(n, generator=g)[:t].int()

    def views(self, buf):
        q = buf[:, :self.hq * self.d].view(self.t, self.hq, self.d)
        return q, buf[:, self.hq * self.d:(self.hq + self.hkv) * self.d].view(self.t, self.hkv, self.d)

    @property
    def pos(self):
        return torch.arange(self.t).int() if self.positions is None else self.positions

    def angles(self):
        at = self.pos.clamp(min=0).long()
        return (self.cos.double()[at], self.sin.double()[at]) if self.rot else (torch.zeros(self.t, 0, dtype=D64),) * 2

    def gpu(self, x):
        return None if x is None else x.to(DEV)

    def table_args(self):
        return (self.gpu(self.cos), self.gpu(self.sin)) if self.rot else (None, None)

    def forward(self, q=None, k=None, q_out=None, k_out=None, stream=None):
        dev = self.qkv.to(DEV)
        q, k = self.views(dev) if q is None else (q, k)
        if q_out is None:
            q_out, k_out = (torch.full((self.t, h, self.d), 7.0, dtype=BF, device=DEV) for h in (self.hq, self.hkv))
        rstd = torch.full((self.t, self.hq + self.hkv), 7.0, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.puro_qk_norm_rope(q, k, self.gpu(self.gains[0]), self.gpu(self.gains[1]), EPS, *self.table_args(),
                            self.gpu(self.positions), self.inter, q_out, k_out, rstd, status, stream)
        return q_out, k_out, rstd, status

    def backward(self, rstd, in_place=False, gains=True, workspace=None):
        q, k = self.views(self.qkv.to(DEV))
        dqo, dko = (x.to(DEV) for x in self.dy)
        dq, dk = (dqo, dko) if in_place else self.views(torch.full_like(self.qkv, 7.0, device=DEV))
        gq, gk = (torch.full((self.d,), 7.0, device=DEV) for _ in range(2)) if gains else (None, None)
        ws = torch.empty(max(4, P.puro_qk_norm_rope_workspace_size(self.t, self.hq, self.hkv, self.d)), dtype=torch.uint8,
                         device=DEV).fill_(255) if gains else None
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.puro_qk_norm_rope_backward(dqo, dko, q, k, rstd, self.gpu(self.gains[0]), self.gpu(self.gains[1]), *self.table_args(),
                                     self.gpu(self.positions), self.inter, dq, dk, gq, gk, ws, status)
        return dq, dk, gq, gk, status


def check_forward(c, out):
    """Half a BF16 step, and the FP32 roundings: rstd at most 2^-20 off (a chain of 8 sums and a tree of at most 7 more, a
    division, a sum, a root and a division, halved by the root), two products and a rotation's three: under 2^-19 of the
    rotated terms' magnitude."""
    cos, sin = c.angles()
    live = (c.pos >= 0)[:, None]
    for x, gain, y, rstd in zip(c.views(c.qkv), c.gains, out[:2], (out[2][:, :c.hq], out[2][:, c.hq:])):
        ref, r, mag = L.qk_forward(x.double(), None if gain is None else gain.double(), cos, sin, c.inter, EPS)
        ref, r, mag = ref * live[..., None], r * live, mag * live[..., None]
        assert bool(((y.cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -19 * mag).all())
        assert bool(((rstd.cpu().double() - r).abs() <= 2.0 ** -20 * r).all())


def check_backward(c, rstd, out):
    """Half a BF16 step and FP32 roundings: the mean's (a chain of 8, a tree of at most 7, a division) and eight more on the
    way to dx, under 2^-18 of the terms' magnitude.  A gain's gradient sums in FP32: at most all terms a thread takes, then
    trees and the blocks' partial sums."""
    cos, sin = c.angles()
    live = (c.pos >= 0)[:, None, None].double()
    groups = 256 // (4 if c.d <= 64 else 8 if c.d <= 128 else 16)
    depth = 2 * -(-c.t * max(c.hq, c.hkv) // groups) + 304 + 40
    for x, dy, gain, r, dx, dg in zip(c.views(c.qkv), c.dy, c.gains, (rstd[:, :c.hq], rstd[:, c.hq:]), out[:2], out[2:4]):
        ref, rg, mag, magg = L.qk_backward(dy.double() * live, x.double(), r.cpu().double(), None if gain is None else gain.double(),
                                           cos, sin, c.inter)
        assert bool(((dx.cpu().double() - ref * live).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -18 * mag).all())
        if dg is not None:
            assert bool(((dg.cpu().double() - rg).abs() <= 2.0 ** -24 * depth * magg + 1e-30).all())


CASES = [(1, 16, 8, 128, 128, False, "arange"), (1, 1, 1, 16, 16, True, "arange"), (3, 5, 1, 64, 32, True, "arange"),
         (37, 12, 2, 128, 64, False, "packed"), (130, 3, 3, 80, 80, False, "shuffled"), (65, 6, 2, 96, 48, True, "packed"),
         (33, 4, 1, 256, 256, False, "shuffled"), (17, 2, 2, 192, 96, False, "arange"), (515, 16, 8, 128, 128, False, "packed"),
         (129, 7, 5, 112, 16, False, "shuffled"), (40, 4, 4, 128, 0, False, "arange"), (2050, 24, 4, 64, 64, False, "packed"),
         (9, 6, 3, 240, 240, True, "shuffled"), (200, 1, 1, 32, 32, False, "packed")]


@pytest.mark.gpu
@pytest.mark.parametrize("gains", [True, False])
@pytest.mark.parametrize("t,hq,hkv,d,rot,inter,positions", CASES)
def test_forward_and_backward(t, hq, hkv, d, rot, inter, positions, gains):
    _need_gpu()
    c = Case(t, hq, hkv, d, rot, inter, positions, gains)
    out = c.forward()
    check_forward(c, out)
    back = c.backward(out[2])
    check_backward(c, out[2], back)
    assert int(out[3]) == 0 and int(back[4]) == 0
    again = c.backward(out[2])
    assert all(torch.equal(a, b) for a, b in zip(back, again))  # sums in a fixed order


@pytest.mark.gpu
def test_in_place_and_head_major_outputs():
    _need_gpu()
    c = Case(70, 6, 2, 128, 128, False, "packed")
    want = c.forward()
    q, k = c.views(c.qkv.to(DEV))
    c.forward(q, k, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    major = [torch.empty(h, c.t, c.d, dtype=BF, device=DEV).transpose(0, 1) for h in (c.hq, c.hkv)]
    c.forward(q_out=major[0], k_out=major[1])
    assert torch.equal(major[0], want[0]) and torch.equal(major[1], want[1])
    plain, inside = c.backward(want[2]), c.backward(want[2], in_place=True)
    assert all(torch.equal(a, b) for a, b in zip(plain, inside))
    assert all(torch.equal(a, b) for a, b in zip(plain[:2], c.backward(want[2], gains=False)[:2]))


@pytest.mark.gpu
def test_the_rest_of_the_buffers_is_left_alone():
    _need_gpu()
    c = Case(9, 2, 1, 64, 64, False)
    rstd = c.forward()[2]
    buf = torch.full((c.t + 2, 6 * c.d), 3.0, dtype=BF, device=DEV)
    c.forward(q_out=buf[1:-1, :2 * c.d].view(c.t, 2, c.d), k_out=buf[1:-1, 3 * c.d:4 * c.d].view(c.t, 1, c.d))
    assert bool((buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, 2 * c.d:3 * c.d] == 3).all() and (buf[:, 4 * c.d:] == 3).all())
    dq, dk = c.backward(rstd)[:2]
    assert bool((dk[:, 0].as_strided((c.t, c.d), (dk.stride(0), 1), dk.storage_offset() + c.d) == 7).all())  # the values' part


@pytest.mark.gpu
def test_nan_in_padding_rows_goes_nowhere():
    _need_gpu()
    c = Case(64, 4, 2, 128, 128, False, "packed")
    bad = c.pos < 0
    c.qkv[bad], c.dy[0][bad], c.dy[1][bad] = float("nan"), float("inf"), float("nan")
    out = c.forward()
    back = c.backward(out[2])
    for x in (*out[:3], *back[:4]):
        assert bool(torch.isfinite(x.float()).all())
    for x in (*out[:3], *back[:2]):
        assert bool((x[bad.to(DEV)] == 0).all())


@pytest.mark.gpu
def test_all_rows_padding():
    _need_gpu()
    c = Case(5, 2, 2, 64, 64, False)
    c.positions = torch.full((5,), -3).int()
    out = c.forward()
    back = c.backward(out[2])
    assert all(bool((x == 0).all()) for x in (*out[:3], *back[:4]))


@pytest.mark.gpu
def test_a_position_past_the_tables_is_reported():
    _need_gpu()
    c = Case(12, 3, 1, 64, 64, False)
    c.positions = torch.arange(12).int()
    ok = c.forward()
    c.positions[7] = c.cos.shape[0]  # the first past the end
    out = c.forward()
    back = c.backward(ok[2])
    assert int(out[3]) == P.PURO_ERR_INVALID_ARG and int(back[4]) == P.PURO_ERR_INVALID_ARG
    rows = torch.arange(12, device=DEV) != 7
    for x, y in zip(out[:3], ok[:3]):
        assert torch.equal(x[rows], y[rows]) and bool(torch.isnan(x[7].float()).all())
    assert bool(torch.isnan(back[0][7].float()).all()) and bool(torch.isfinite(back[0][rows].float()).all())
    assert bool(torch.isnan(back[2]).all())


@pytest.mark.gpu
def test_offsets_past_32_bits():
    _need_gpu()
    c = Case(4, 2, 1, 64, 64, False)
    stride = 2 ** 30 + 8
    buf = torch.empty(3 * stride + 4 * 64, dtype=BF, device=DEV)  # 6.4 GB
    q = buf.as_strided((4, 2, 64), (stride, 64, 1))
    k = buf.as_strided((4, 1, 64), (stride, 64, 1), 128)
    want = c.forward()
    for dst, src in zip((q, k), c.views(c.qkv)):
        dst.copy_(src)
    got = c.forward(q, k, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(got[2], want[2])


@pytest.mark.gpu
def test_captured_calls_and_another_stream():
    _need_gpu()
    c = Case(300, 12, 2, 128, 128, False, "packed")
    want = c.forward()
    wantb = c.backward(want[2])
    q, k = c.views(c.qkv.to(DEV))
    args = [c.gpu(x) for x in (*c.gains, c.cos, c.sin, c.positions)]
    qo, ko, rstd = (torch.zeros_like(x) for x in want[:3])
    dqo, dko = (x.to(DEV) for x in c.dy)
    dq, dk = torch.zeros_like(qo), torch.zeros_like(ko)
    gq, gk = torch.zeros(c.d, device=DEV), torch.zeros(c.d, device=DEV)
    ws = torch.empty(P.puro_qk_norm_rope_workspace_size(c.t, c.hq, c.hkv, c.d), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()

    def both(stream=None):
        P.puro_qk_norm_rope(q, k, args[0], args[1], EPS, args[2], args[3], args[4], False, qo, ko, rstd, stream=stream)
        P.puro_qk_norm_rope_backward(dqo, dko, q, k, rstd, args[0], args[1], args[2], args[3], args[4], False, dq, dk, gq, gk, ws,
                                     stream=stream)

    def check():
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((qo, ko, rstd, dq, dk, gq, gk), (*want[:3], *wantb[:4])))
        for x in (qo, ko, rstd, dq, dk, gq, gk):
            x.zero_()
        torch.cuda.synchronize()

    both(side)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(2):
        graph.replay()
        check()


# ------------------------------------------------------------- refusals, without a GPU
def _h(heads=2, data=A, ts=256, hs=64, reserved=0):
    return P.puro_heads_t(data, ts, hs, heads, reserved)


def _fwd(lib, q=_h(), k=_h(1), tokens=4, d=64, gq=A, gk=A, eps=EPS, cos=A, sin=A, n=16, rot=64, pos=A, qo=_h(), ko=_h(1), rstd=A,
         status=None):
    r = ctypes.byref
    return lib.puro_qk_norm_rope(r(q), r(k), tokens, d, gq, gk, eps, cos, sin, n, rot, 0, pos, r(qo), r(ko), rstd, status, None)


def test_refusals():
    lib = P.load_library()
    bad = P.PURO_ERR_INVALID_ARG
    for kw in (dict(d=8), dict(d=72), dict(d=272), dict(rot=8), dict(rot=80), dict(rot=-16), dict(tokens=-1), dict(eps=-1.0),
               dict(eps=float("nan")), dict(cos=None), dict(sin=A + 4), dict(n=-1), dict(pos=None, n=3), dict(pos=A + 2),
               dict(gq=A + 2), dict(rstd=A + 1), dict(status=A + 2), dict(q=_h(data=None)), dict(q=_h(data=A + 8)),
               dict(q=_h(ts=257)), dict(q=_h(hs=-8)), dict(q=_h(heads=-1)), dict(q=_h(reserved=1)), dict(qo=_h(heads=3)),
               dict(qo=_h(hs=56)), dict(qo=_h(ts=0)), dict(ko=_h(0))):
        assert _fwd(lib, **kw) == bad, kw
    assert _fwd(lib, tokens=2 ** 31) == P.PURO_ERR_UNSUPPORTED
    assert _fwd(lib, tokens=0) == P.PURO_OK
    assert _fwd(lib, q=_h(0), k=_h(0), qo=_h(0), ko=_h(0)) == P.PURO_OK


def _bwd(lib, dqo=_h(), dko=_h(1), q=_h(), k=_h(1), rstd=A, tokens=4, d=64, dq=_h(), dk=_h(1), gq=A, gk=A, ws=A, nbytes=1 << 20):
    r = ctypes.byref
    return lib.puro_qk_norm_rope_backward(r(dqo), r(dko), r(q), r(k), rstd, tokens, d, A, A, A, A, 16, 64, 0, A, r(dq), r(dk), gq,
                                          gk, ws, nbytes, None, None)


def test_backward_refusals():
    lib = P.load_library()
    bad = P.PURO_ERR_INVALID_ARG
    need = P.puro_qk_norm_rope_workspace_size(4, 2, 1, 64)
    assert need > 0
    for kw in (dict(rstd=None), dict(ws=None), dict(ws=A + 2), dict(nbytes=need - 1), dict(gq=A + 2), dict(dq=_h(hs=0)),
               dict(dq=_h(3)), dict(dko=_h(2)), dict(d=24), dict(q=_h(data=A + 2))):
        assert _bwd(lib, **kw) == bad, kw
    assert _bwd(lib, tokens=0, gq=None, gk=None, ws=None, nbytes=0) == P.PURO_OK


def test_workspace_is_one_partial_sum_a_block():
    for t, hq, hk, d in ((1, 16, 8, 128), (8192, 16, 8, 128), (5003, 12, 2, 128), (10 ** 6, 1, 64, 256), (7, 0, 3, 16)):
        n = P.puro_qk_norm_rope_workspace_size(t, hq, hk, d)
        assert n % (4 * d) == 0 and 0 < n // (4 * d) <= 304
    assert P.puro_qk_norm_rope_workspace_size(0, 4, 4, 64) == 0


def test_python_refusals():
    q = torch.zeros(4, 2, 64, dtype=BF)
    with pytest.raises(ValueError):  # not on the GPU
        P._heads(q, "q", 4, 64)
    with pytest.raises(ValueError):
        P._sized(torch.zeros(5), torch.float32, 4, "rstd")
    with pytest.raises(ValueError):
        P._tables(torch.zeros(4, 2), torch.zeros(4, 3))
    with pytest.raises(ValueError):
        P._tables(torch.zeros(4, 2), None)
