"""A decoder layer's training step from the public calls: RMSNorm + quantise, the
qkv linear with its bias, query and key norms with the rotation, attention (plain
torch: not part of this library), the output projection onto the residual stream,
the gated MLP, and all of it backwards.

Whole-layer values are compared with autograd in 64 bits on the unquantised layer.
E4M3's half step is 2^-4 of a value, 0.027 of a random tensor's norm once rounded;
a product of two such operands is then 0.038 off, and the longest chain here goes
through nine of them (four forward, whose outputs the backward reads, five
backward): 0.12 if their errors are independent.  The bound is twice that.  What
each call does exactly is tested call by call elsewhere; here it is that they fit
together, also captured into a graph."""
import pytest
import torch

import paper_2608_27370_gb300 as P

DEV, BF, D64, u8 = "cuda", torch.bfloat16, torch.float64, torch.uint8
M, SEQ, H, HQ, HK, D, F, EPS = 256, 128, 256, 4, 2, 64, 384, 1e-6
QKV = (HQ + 2 * HK) * D
OFF = 2 * (9 ** 0.5) * 0.038


def _normal(shape, std, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(BF)


def _weights():
    return {"qkv": _normal((QKV, H), 0.06, 1), "o": _normal((H, HQ * D), 0.06, 2), "gu": _normal((2 * F, H), 0.06, 3),
            "down": _normal((H, F), 0.06, 4), "bias": _normal((QKV,), 0.2, 5), "qg": 1 + _normal((D,), 0.2, 6), "kg": 1 + _normal((D,), 0.2, 7),
            "n1": 1 + _normal((H,), 0.1, 8), "n2": 1 + _normal((H,), 0.1, 9)}


def _tables(dtype):
    a = torch.arange(SEQ, dtype=D64, device=DEV)[:, None] * 1e4 ** (-2 * torch.arange(D // 2, dtype=D64, device=DEV) / D)
    return a.cos().to(dtype), a.sin().to(dtype)


def _attention(q, k, v):
    """Causal, by sequence; heads of the queries share those of the keys."""
    sh = lambda x: x.view(M // SEQ, SEQ, -1, D).transpose(1, 2)  # noqa: E731
    q, k, v = sh(q), sh(k).repeat_interleave(HQ // HK, 1), sh(v).repeat_interleave(HQ // HK, 1)
    s = (q @ k.transpose(-1, -2)) / D ** 0.5
    s = s.masked_fill(torch.ones(SEQ, SEQ, dtype=torch.bool, device=DEV).triu(1), float("-inf"))
    return (s.softmax(-1) @ v).transpose(1, 2).reshape(M, HQ * D)


def _norm(x, g):
    return x * (x.pow(2).mean(-1, keepdim=True) + EPS) ** -0.5 * g


def _reference(h, w):
    """The layer in the type of its inputs."""
    cos, sin = (t.repeat(M // SEQ, 1)[:, None] for t in _tables(h.dtype))
    turn = lambda x: torch.cat([x[..., :D // 2] * cos - x[..., D // 2:] * sin, x[..., D // 2:] * cos + x[..., :D // 2] * sin], -1)  # noqa: E731
    qkv = (_norm(h, w["n1"]) @ w["qkv"].t() + w["bias"]).view(M, HQ + 2 * HK, D)
    a = _attention(turn(_norm(qkv[:, :HQ], w["qg"])), turn(_norm(qkv[:, HQ:HQ + HK], w["kg"])), qkv[:, HQ + HK:])
    h2 = h + a @ w["o"].t()
    gu = _norm(h2, w["n2"]) @ w["gu"].t()
    return h2 + (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ w["down"].t()


class Layer:
    """The buffers a program keeps, and the step's calls."""

    def __init__(self, w):
        self.w = w
        e = lambda *s, dtype=BF: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
        op = lambda r, c, role=P.ROLE_ACT: P.FP8Operand(e(r, c, dtype=u8), P.empty_scales(r, c, P.SCALE_BLOCK, role, DEV), role=role)  # noqa: E731
        both = lambda r, c: P.Quantized(op(r, c), op(c, r))  # noqa: E731
        self.wq = {n: P.quantize(w[n], P.E4M3, P.SCALE_BLOCK, P.ROLE_WEIGHT) for n in ("qkv", "o", "gu", "down")}
        self.x1, self.x2, self.a8, self.hid = both(M, H), both(M, H), both(M, HQ * D), both(M, F)
        self.d8, self.g8, self.o8, self.q8 = both(M, H), both(M, 2 * F), both(M, H), both(M, QKV)
        self.r1, self.r2 = e(M, dtype=torch.float32), e(M, dtype=torch.float32)
        self.qkv, self.qk_out, self.h2, self.gate_up, self.out = e(M, QKV), e(M, (HQ + HK) * D), e(M, H), e(M, 2 * F), e(M, H)
        self.rstd = e(M, HQ + HK, dtype=torch.float32)
        self.cos, self.sin = _tables(torch.float32)
        self.pos = torch.arange(SEQ, device=DEV, dtype=torch.int32).repeat(M // SEQ)
        self.dhid, self.dn2, self.da, self.dqkv, self.dn1 = e(M, F), e(M, H), e(M, HQ * D), e(M, QKV), e(M, H)
        self.dw = {n: e(*w[n].shape) for n in ("qkv", "o", "gu", "down")}
        self.dbias, self.dqg, self.dkg = (e(n, dtype=torch.float32) for n in (QKV, D, D))
        self.ws = e(max(P.puro_act_backward_workspace_size(M, QKV), P.puro_qk_norm_rope_workspace_size(M, HQ, HK, D)), dtype=u8)
        self.st = torch.zeros(1, dtype=torch.int32, device=DEV)

    @staticmethod
    def copies(q):
        return q.rowwise.data, q.rowwise.scale, q.colwise.data, q.colwise.scale

    @staticmethod
    def split(x, heads):
        """Query, key and (where there are any) value heads of a fused row."""
        v = x.view(M, -1, D)
        return v[:, :HQ], v[:, HQ:HQ + HK], v[:, HQ + HK:heads]

    def forward(self, h):
        w, st = self.w, self.st
        P.puro_fp8_quantize_rmsnorm(h, w["n1"], EPS, P.E4M3, self.r1, None, *self.copies(self.x1), st)
        P.puro_fp8_linear_fprop_epilogue(self.x1.rowwise, self.wq["qkv"].rowwise, self.qkv, w["bias"], dev_status=st)
        q, k, v = self.split(self.qkv, HQ + 2 * HK)
        qo, ko, _ = self.split(self.qk_out, HQ + HK)
        P.puro_qk_norm_rope(q, k, w["qg"], w["kg"], EPS, self.cos, self.sin, self.pos, False, qo, ko, self.rstd, st)
        self.a = _attention(qo.float(), ko.float(), v.float()).to(BF)
        P.quantize(self.a, out=self.a8, dev_status=st)
        P.puro_fp8_linear_fprop_epilogue(self.a8.rowwise, self.wq["o"].rowwise, self.h2, residual=h, dev_status=st)
        P.puro_fp8_quantize_rmsnorm(self.h2, w["n2"], EPS, P.E4M3, self.r2, None, *self.copies(self.x2), st)
        P.puro_fp8_gated_fprop(self.x2.rowwise, self.wq["gu"].rowwise, P.ACT_SILU, P.E4M3, self.gate_up, None, *self.copies(self.hid), st)
        P.puro_fp8_linear_fprop_epilogue(self.hid.rowwise, self.wq["down"].rowwise, self.out, residual=self.h2, dev_status=st)
        return self.out

    def linear_backward(self, d8, name, dx, x8):
        P.puro_fp8_linear_backward(d8.rowwise, self.wq[name].colwise, dx, d8.colwise, x8.colwise, self.dw[name], dev_status=self.st)

    @staticmethod
    def norm_backward(dn, h, rstd, g):  # (not part of this library)
        x, d = h.float() * rstd[:, None], dn.float() * g.float()
        return rstd[:, None] * (d - x * (d * x).mean(-1, keepdim=True))

    def backward(self, dout, h):
        w, st = self.w, self.st
        P.quantize(dout, out=self.d8, dev_status=st)
        self.linear_backward(self.d8, "down", self.dhid, self.hid)
        P.puro_fp8_quantize_gated_backward(self.dhid, self.gate_up[:, :F], self.gate_up[:, F:], P.ACT_SILU, P.E4M3, None, *self.copies(self.g8), st)
        self.linear_backward(self.g8, "gu", self.dn2, self.x2)
        dh2 = dout.float() + self.norm_backward(self.dn2, self.h2, self.r2, w["n2"])
        P.quantize(dh2.to(BF), out=self.o8, dev_status=st)
        self.linear_backward(self.o8, "o", self.da, self.a8)
        qo, ko, _ = self.split(self.qk_out, HQ + HK)
        q, k, v = self.split(self.qkv, HQ + 2 * HK)
        dq, dk, dv = self.split(self.dqkv, HQ + 2 * HK)
        with torch.enable_grad():
            leaves = [t.detach().float().requires_grad_() for t in (qo, ko, v)]
            gq, gk, gv = torch.autograd.grad(_attention(*leaves), leaves, self.da.float())
        dv.copy_(gv)
        P.puro_qk_norm_rope_backward(gq.to(BF), gk.to(BF), q, k, self.rstd, w["qg"], w["kg"], self.cos, self.sin, self.pos, False, dq, dk,
                                     self.dqg, self.dkg, self.ws, st)
        P.puro_fp8_quantize_act_backward(self.dqkv, None, P.ACT_NONE, P.E4M3, None, self.dbias, self.ws, *self.copies(self.q8), st)
        self.linear_backward(self.q8, "qkv", self.dn1, self.x1)
        return (dh2 + self.norm_backward(self.dn1, h, self.r1, w["n1"])).to(BF)

    def results(self):
        return {"out": self.out, "bias": self.dbias, "qg": self.dqg, "kg": self.dkg, **self.dw}


@pytest.mark.gpu
def test_a_layer_forward_backward_and_captured():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    w, h, dout = _weights(), _normal((M, H), 1.0, 20), _normal((M, H), 1e-2, 21)
    layer = Layer(w)
    layer.forward(h)
    dh = layer.backward(dout, h)
    assert int(layer.st) == 0
    got = {**layer.results(), "h": dh}
    got = {n: t.clone() for n, t in got.items()}

    leaves = {n: t.double().requires_grad_() for n, t in w.items()}
    h64 = h.double().requires_grad_()
    out = _reference(h64, leaves)
    names = ["qkv", "o", "gu", "down", "bias", "qg", "kg"]
    grads = torch.autograd.grad(out, [leaves[n] for n in names] + [h64], dout.double())
    ref = {"out": out.detach(), **dict(zip(names + ["h"], grads))}
    for n, t in got.items():
        off = float((t.double() - ref[n]).norm() / ref[n].norm())
        assert off < OFF, f"{n}: {off:.3f}"

    # the same calls again, and captured: the same bytes
    layer.forward(h)
    layer.backward(dout, h)
    assert all(torch.equal(t, got[n]) for n, t in layer.results().items())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(h)
        layer.backward(dout, h)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, got[n]) for n, t in layer.results().items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(h)
        layer.backward(dout, h)
    for t in layer.results().values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, got[n]) for n, t in layer.results().items())


@pytest.mark.gpu
def test_one_token_at_a_time_in_bf16():
    """The same layer's linears, norms and rotation on one token after another give the rows of the whole batch."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    w, h = _weights(), _normal((24, H), 1.0, 30)
    cos, sin = _tables(torch.float32)
    e = lambda *s: torch.empty(s, dtype=BF, device=DEV)  # noqa: E731

    def step(x, pos):
        n = x.shape[0]
        qkv, qo, ko, hid, out = e(n, QKV), e(n, HQ, D), e(n, HK, D), e(n, F), e(n, H)
        P.puro_bf16_linear_fprop_epilogue(x, w["qkv"], qkv, w["bias"])
        q, k = qkv.view(n, -1, D)[:, :HQ], qkv.view(n, -1, D)[:, HQ:HQ + HK]
        P.puro_qk_norm_rope(q, k, w["qg"], w["kg"], EPS, cos, sin, pos, False, qo, ko)
        P.puro_bf16_gated_fprop(x, w["gu"], P.ACT_SILU, None, hid)
        P.puro_bf16_linear_fprop_epilogue(hid, w["down"], out, residual=x)
        return qkv, qo, ko, hid, out

    pos = torch.arange(24, dtype=torch.int32, device=DEV)
    whole = step(h, pos)
    for i in range(24):
        one = step(h[i:i + 1], pos[i:i + 1])
        for a, b in zip(one, whole):
            # both round the same products once; the sums' orders differ: a BF16 step at most, or what cancelled
            d = (a[0].double() - b[i].double()).abs()
            assert bool((d <= 2.0 ** -7 * b[i].double().abs() + 2.0 ** -9 * b[i].double().pow(2).mean().sqrt()).all())


@pytest.mark.gpu
def test_a_residual_stream_updated_in_place():
    """Each linear adds to the stream in place and the next kernel, already started, reads it: captured and replayed, the
    bytes of calls that are waited for one by one.  (Rows end inside a 32-byte sector.)"""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    width, inner, blocks, rows = 1032, 520, 12, 3
    w_in = [_normal((inner, width), width ** -0.5, 40 + i) for i in range(blocks)]
    w_out = [_normal((width, inner), inner ** -0.5, 60 + i) for i in range(blocks)]
    h0, h, mid = _normal((rows, width), 1.0, 80), torch.empty((rows, width), dtype=BF, device=DEV), torch.empty(
        (rows, inner), dtype=BF, device=DEV)

    def run(wait):
        h.copy_(h0)
        for wi, wo in zip(w_in, w_out):
            P.puro_bf16_linear_fprop_epilogue(h, wi, mid, act=P.ACT_GELU)
            wait()
            P.puro_bf16_linear_fprop_epilogue(mid, wo, h, residual=h)
            wait()

    run(torch.cuda.synchronize)
    ref = h.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(lambda: None)
    for _ in range(20):
        graph.replay()
        assert torch.equal(h, ref)
