"""The references of _layer_ops.py: gradients against differences, activations against torch's own."""
import pytest
import torch

import _layer_ops as L

D64 = torch.float64


def _angles(t, rot):
    a = torch.rand(t, rot // 2, dtype=D64) * 6.3
    return a.cos(), a.sin()


@pytest.mark.parametrize("rot,inter", [(16, False), (16, True), (0, False), (32, False)])
def test_qk_gradients_are_the_differences(rot, inter):
    torch.manual_seed(rot + inter)
    x, gain, dy = torch.randn(3, 2, 32, dtype=D64), 1 + 0.2 * torch.randn(32, dtype=D64), torch.randn(3, 2, 32, dtype=D64)
    cos, sin = _angles(3, rot)
    f = lambda x, g: (L.qk_forward(x, g, cos, sin, inter, 1e-6)[0] * dy).sum()  # noqa: E731
    dx, dg, _, _ = L.qk_backward(dy, x, L.qk_forward(x, gain, cos, sin, inter, 1e-6)[1], gain, cos, sin, inter)
    h = 1e-6  # a central difference is off by O(h^2) + 2^-52 |f| / h: below 1e-8
    for grad, at in ((dx, 0), (dg, 1)):
        for i in range(0, grad.numel(), 7):
            p = [x.clone(), gain.clone()], [x.clone(), gain.clone()]
            p[0][at].view(-1)[i] += h
            p[1][at].view(-1)[i] -= h
            diff = (f(*p[0]) - f(*p[1])) / (2 * h)
            assert abs(float(diff - grad.view(-1)[i])) < 1e-7


def test_rotation_keeps_lengths_and_its_transpose_undoes_it():
    torch.manual_seed(0)
    x = torch.randn(5, 3, 64, dtype=D64)
    cos, sin = _angles(5, 32)
    for inter in (False, True):
        y = L.rotate(x, cos, sin, inter)
        assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1), rtol=1e-14)
        assert torch.allclose(L.rotate(y, cos, sin, inter, back=True), x, rtol=0, atol=1e-14)
        assert torch.equal(y[..., 32:], x[..., 32:])


def test_neighbouring_pairs_are_the_half_split_ones_in_another_order():
    torch.manual_seed(1)
    x = torch.randn(4, 2, 16, dtype=D64)
    cos, sin = _angles(4, 16)
    order = torch.cat([torch.arange(0, 16, 2), torch.arange(1, 16, 2)])
    assert torch.equal(L.rotate(x, cos, sin, True)[..., order], L.rotate(x[..., order], cos, sin, False))


@pytest.mark.parametrize("kind", L.ACTS)
def test_slopes_are_the_differences(kind):
    z = torch.linspace(-12, 12, 1001, dtype=D64) + 1e-3
    h = 1e-6
    diff = (L.act(z + h, kind) - L.act(z - h, kind)) / (2 * h)
    assert float((diff - L.slope(z, kind)).abs().max()) < 1e-8


def test_activations_are_torchs():
    z = torch.linspace(-8, 8, 333, dtype=D64)
    F = torch.nn.functional
    for kind, ref in (("silu", F.silu(z)), ("gelu", F.gelu(z)), ("gelu_tanh", F.gelu(z, approximate="tanh")), ("relu", F.relu(z))):
        assert torch.allclose(L.act(z, kind), ref, rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("kind", L.ACTS[1:])
def test_gate_gradients_are_the_differences(kind):
    torch.manual_seed(3)
    g, u, dh = (torch.randn(64, dtype=D64) for _ in range(3))
    dg, du = L.gated_backward(dh, g, u, kind)
    h = 1e-6
    f = lambda g, u: L.gated(g, u, kind) * dh  # noqa: E731
    assert float(((f(g + h, u) - f(g - h, u)) / (2 * h) - dg).abs().max()) < 1e-8
    assert float(((f(g, u + h) - f(g, u - h)) / (2 * h) - du).abs().max()) < 1e-8
