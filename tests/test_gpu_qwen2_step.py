"""The training step of a layer without query and key norms, from the public calls: the
qkv linear with its bias, the rotation of its output in place, backwards through the
rotation into the qkv linear's main gradient, the Muon directions of that gradient
and another's, the MuonH step along them, the weights quantised anew.  Each result is
compared with 64 bits of what its call was given; and the whole step, captured into
a graph and replayed, with the calls one by one."""
import math

import pytest
import torch

import _muon as M
import _rope as R
import paper_2608_27370_gb300 as P

pytestmark = pytest.mark.gpu
DEV, BF, F32, u8 = "cuda", torch.bfloat16, torch.float32, torch.uint8
T, H, HQ, HK, D, F = 384, 256, 6, 2, 64, 640
QKV = (HQ + 2 * HK) * D
ETA = 0.02


def _normal(shape, std, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std)


class Step:
    def __init__(self):
        e = lambda *s, dtype=BF: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
        op = lambda r, c, role=P.ROLE_ACT: P.FP8Operand(e(r, c, dtype=u8), P.empty_scales(r, c, P.SCALE_BLOCK, role, DEV), role=role)  # noqa: E731
        both = lambda r, c, role=P.ROLE_ACT: P.Quantized(op(r, c, role), op(c, r, role))  # noqa: E731
        self.x = _normal((T, H), 1.0, 1).to(BF).to(DEV)
        self.bias = _normal((QKV,), 0.2, 2).to(BF).to(DEV)
        self.dy = _normal((T, QKV), 1e-3, 3).to(BF).to(DEV)
        self.w = [_normal((QKV, H), 0.05, 4).to(DEV), _normal((H, F), 0.05, 5).to(DEV)]  # qkv, down: master weights
        self.radius = [float(w.double().norm()) for w in self.w]
        self.wb = [w.to(BF) for w in self.w]
        self.wq = [both(*w.shape, role=P.ROLE_WEIGHT) for w in self.w]
        self.main = [torch.zeros_like(self.w[0]), _normal((H, F), 1e-3, 6).to(DEV)]
        self.mom = [_normal(w.shape, 3e-3, 7 + i).to(DEV) for i, w in enumerate(self.w)]
        self.u = [torch.empty_like(w) for w in self.w]
        self.xq, self.dq = both(T, H), both(T, QKV)
        self.qkv, self.dqkv, self.dx = e(T, QKV), e(T, QKV), e(T, H)
        self.freq = P.rope_frequencies(D, 1e6, P.ROPE_TURNS, 4.0, 32768, device=DEV)
        self.scale = 0.1 * math.log(4.0) + 1
        self.pos = torch.cat([torch.arange(200), torch.arange(150), torch.full((34,), -1)]).int().to(DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.table = P.muon_table(list(zip(self.main, self.mom, self.u)))
        self.ws = e(P.puro_muon_direction_workspace_size(self.table), dtype=u8)
        self.mats = list(zip(self.w, self.u, self.wb, self.radius))
        self.hws = e(P.puro_muonh_grouped_workspace_size(self.mats), dtype=u8)
        self.sums = e(2, 3, dtype=torch.float64)
        self.weights = P.weight_table(list(zip(self.wb, self.wq)))
        P.puro_fp8_quantize_weights(self.weights)

    @staticmethod
    def heads(x):
        v = x.view(T, HQ + 2 * HK, D)
        return v[:, :HQ], v[:, HQ:HQ + HK]

    def forward(self):
        P.quantize(self.x, out=self.xq, dev_status=self.status)
        P.puro_fp8_linear_fprop_epilogue(self.xq.rowwise, self.wq[0].rowwise, self.qkv, self.bias, dev_status=self.status)
        q, k = self.heads(self.qkv)
        P.puro_rope(q, k, self.freq, self.pos, False, q, k, scale=self.scale)

    def backward(self):
        self.dqkv.copy_(self.dy)
        q, k = self.heads(self.dqkv)
        P.puro_rope_backward(q, k, self.freq, self.pos, False, q, k, scale=self.scale)
        P.quantize(self.dqkv, out=self.dq, dev_status=self.status)
        self.main[0].zero_()
        P.puro_fp8_linear_wgrad_main_grad(self.dq.colwise, self.xq.colwise, self.main[0], dev_status=self.status)

    def update(self):
        P.puro_muon_direction_grouped(self.table, self.ws, dev_status=self.status)
        P.puro_muonh_step_grouped(self.mats, ETA, self.sums, self.hws)
        P.puro_fp8_quantize_weights(self.weights, dev_status=self.status)

    def run(self):
        self.forward()
        self.backward()
        self.update()

    def state(self):
        return [self.qkv, self.dqkv, *self.main, *self.mom, *self.u, *self.w, *self.wb] + \
            [t for q in self.wq for t in (q.rowwise.data, q.rowwise.scale, q.colwise.data, q.colwise.scale)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def test_each_call_of_the_step_against_64_bits():
    s, before = Step(), Step()
    q, k = s.heads(before.qkv)  # the linear's output without the rotation
    P.quantize(s.x, out=s.xq)
    P.puro_fp8_linear_fprop_epilogue(s.xq.rowwise, s.wq[0].rowwise, before.qkv, s.bias)
    s.run()
    torch.cuda.synchronize()
    assert int(s.status) == 0
    scale = float(torch.tensor(s.scale))
    for got, x, back in ((s.qkv, before.qkv, False), (s.dqkv, s.dy, True)):
        for y, v in zip(s.heads(got), s.heads(x)):
            want, mag, off = R.rotation(v.cpu(), s.freq.cpu(), s.pos.tolist(), False, scale, back)
            err = (y.cpu().double() - want).abs()
            assert (err <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * mag + 2.0 ** -19 * off + 2.0 ** -133).all()
        assert torch.equal(got.view(T, -1, D)[:, HQ + HK:], x.view(T, -1, D)[:, HQ + HK:])  # the values are not turned
    for i in range(2):
        m, v = M.update(s.main[i].cpu().double(), before.mom[i].cpu().double(), float(torch.tensor(0.95)), True)
        assert ((s.mom[i].cpu().double() - m).abs() <= 2.0 ** -24 * m.abs()).all()
        want, bound = M.bound(v, F32)
        assert float((s.u[i].cpu().double() - want).norm()) <= bound
        # the hyperball step along u, and what it leaves
        w0, u, radius = before.w[i].cpu().double(), s.u[i].cpu().double(), s.radius[i]
        w1 = w0 - ETA * radius * u / u.norm()
        w1 = radius * w1 / w1.norm()
        err = (s.w[i].cpu().double() - w1).abs()
        assert (err <= 1e-5 * w1.abs() + 1e-6 * w1.pow(2).mean().sqrt()).all()  # (as in the step's own test)
        assert torch.equal(s.wb[i], s.w[i].to(BF))
        again = P.quantize(s.wb[i], P.E4M3, P.SCALE_BLOCK, P.ROLE_WEIGHT)
        assert torch.equal(again.rowwise.data, s.wq[i].rowwise.data) and torch.equal(again.colwise.data, s.wq[i].colwise.data)


def test_the_step_in_a_graph():
    eager, graphed = Step(), Step()
    eager.run()  # (and once ahead of the capture: modules load at their first call)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.run()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager.state(), graphed.state()):
        assert torch.equal(a, b)
    for _ in range(2):
        eager.run()
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager.state(), graphed.state()):
        assert torch.equal(a, b)
    assert int(graphed.status) == 0
