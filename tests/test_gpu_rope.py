"""The position rotation without a norm, its backward and its tables, against 64 bits (_rope.py)."""
import math

import pytest
import torch

import _rope as R
import paper_2608_27370_gb300 as P

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16
KINDS = {"none": P.ROPE_NONE, "linear": P.ROPE_LINEAR, "base": P.ROPE_BASE, "turns": P.ROPE_TURNS, "index": P.ROPE_INDEX}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def check(y, x, freq, positions, inter, scale=1.0, back=False):
    """Half a BF16 step, the roundings of the FP32 products and of the scaled cosine (4 half steps of the magnitude), and cosines and
    sines that are 2^-19 off."""
    want, mag, off = R.rotation(x.cpu(), freq.cpu(), positions, inter, scale, back)
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -22 * mag + 2.0 ** -19 * off + 2.0 ** -133
    err = (y.cpu().double() - want).abs()
    assert (err <= bound).all(), float((err / bound).max())


def qkv_views(t, hq, hkv, d, seed=0):
    g = torch.Generator().manual_seed(seed + t + 100 * d)
    qkv = (torch.randn(t, (hq + 2 * hkv) * d, generator=g) * torch.exp2(torch.randint(-3, 4, (t, 1), generator=g))).to(BF).to(DEV)
    return qkv, qkv[:, :hq * d].view(t, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d)


CASES = [(1, 1, 1, 16, 16, False), (1, 12, 2, 128, 128, False), (7, 3, 1, 64, 32, True), (33, 5, 2, 80, 32, False), (129, 12, 2, 128, 64, True),
         (65, 4, 4, 96, 96, False), (50, 9, 3, 192, 192, True), (257, 2, 1, 256, 256, False), (31, 6, 5, 256, 16, True), (1000, 1, 7, 48, 48, False)]


@pytest.mark.parametrize("t,hq,hkv,d,rot,inter", CASES)
@pytest.mark.parametrize("call", ["forward", "backward"])
def test_against_64_bits(t, hq, hkv, d, rot, inter, call):
    _, q, k = qkv_views(t, hq, hkv, d)
    freq = P.rope_frequencies(rot, 1e4)
    g = torch.Generator().manual_seed(t)
    pos = torch.randint(0, 5000, (t,), generator=g, dtype=torch.int32)
    pos[t // 2] = -1 if t > 2 else 77
    qo, ko = (torch.full((t, h, d), 7.0, dtype=BF, device=DEV) for h in (hq, hkv))
    fn = P.puro_rope if call == "forward" else P.puro_rope_backward
    fn(q, k, freq, pos.to(DEV), inter, qo, ko)
    for x, y in ((q, qo), (k, ko)):
        check(y, x, freq, pos.tolist(), inter, back=call == "backward")


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_scaled_frequencies_and_the_scale(kind):
    t, d = 40, 128
    _, q, k = qkv_views(t, 4, 2, d)
    freq = P.rope_frequencies(d, 1e6, KINDS[kind], 8.0, 32768)
    scale = 0.1 * math.log(8.0) + 1
    pos = [2 ** 31 - 1, 2 ** 30 + 3, 262143, 1000003] + list(range(36))
    p = torch.tensor(pos, dtype=torch.int32, device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    P.puro_rope(q, k, freq, p, False, qo, ko, scale=scale)
    check(qo, q, freq, pos, False, float(torch.tensor(scale)))
    check(ko, k, freq, pos, False, float(torch.tensor(scale)))


def test_positions_by_default_and_one_kind_of_heads():
    _, q, k = qkv_views(19, 3, 2, 64)
    freq = P.rope_frequencies(64, 1e4)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    P.puro_rope(q, None, freq, None, False, qo, None)
    P.puro_rope(None, k, freq, None, False, None, ko)
    check(qo, q, freq, range(19), False)
    check(ko, k, freq, range(19), False)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [32, 128])
def test_in_place_and_beside_the_heads(inter, rot):
    """In place in the qkv output: what lies beside the heads stays, and the result is that of the call out of place."""
    qkv, q, k = qkv_views(37, 5, 2, 128)
    freq, before = P.rope_frequencies(rot, 1e4), qkv.clone()
    pos = torch.arange(37, dtype=torch.int32, device=DEV)
    pos[-5:] = -1
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    P.puro_rope(q, k, freq, pos, inter, qo, ko)
    P.puro_rope(q, k, freq, pos, inter, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(qkv[:, 7 * 128:], before[:, 7 * 128:])


def test_heads_ahead_of_tokens_and_wide_strides():
    t, h, d = 21, 3, 64
    x = torch.randn(h, t, d, device=DEV).to(BF).transpose(0, 1)
    y = torch.full((t, 2 * h, d + 8), 5.0, dtype=BF, device=DEV)
    freq = P.rope_frequencies(64, 1e4)
    P.puro_rope(x, None, freq, None, True, y[:, ::2, :d], None)
    check(y[:, ::2, :d], x, freq, range(t), True)
    assert (y[:, 1::2] == 5).all() and (y[:, ::2, d:] == 5).all()


def test_padding_rows_are_zero_whatever_they_hold():
    _, q, k = qkv_views(12, 4, 2, 96)
    q[3:5], k[3:5] = float("nan"), float("inf")
    freq = P.rope_frequencies(96, 1e4)
    pos = list(range(12))
    pos[3], pos[4] = -1, -(2 ** 31)
    p = torch.tensor(pos, dtype=torch.int32, device=DEV)
    for fn in (P.puro_rope, P.puro_rope_backward):
        qo, ko = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
        fn(q, k, freq, p, False, qo, ko)
        for y in (qo, ko):
            assert (y[3:5].view(torch.int16) == 0).all() and torch.isfinite(y).all()


def test_non_finite_channels_stay_in_their_pair():
    _, q, k = qkv_views(6, 2, 1, 64)
    q[2, 1, 5], q[4, 0, 63] = float("inf"), float("nan")
    freq = P.rope_frequencies(64, 1e4)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    P.puro_rope(q, k, freq, None, False, qo, ko)
    bad = ~torch.isfinite(qo)
    assert bad[2, 1, [5, 37]].all() and bad[4, 0, [31, 63]].all() and int(bad.sum()) == 4


@pytest.mark.parametrize("inter", [False, True])
def test_the_backward_is_the_transpose_and_the_differences(inter):
    """<R x, y> = <x, R^T y> for the calls themselves, up to their roundings; and R^T y against differences of the loss, which is linear."""
    t, h, d, scale = 9, 2, 64, 1.25
    _, x, _ = qkv_views(t, h, 1, d)
    y = torch.randn(t, h, d, device=DEV).to(BF)
    freq, pos = P.rope_frequencies(32, 1e4), torch.arange(t, dtype=torch.int32, device=DEV) * 17
    rx, ry = torch.empty_like(y), torch.empty_like(y)
    P.puro_rope(x, None, freq, pos, inter, rx, None, scale=scale)
    P.puro_rope_backward(y, None, freq, pos, inter, ry, None, scale=scale)
    a, b = rx.double() * y.double(), x.double() * ry.double()
    bound = 2.0 ** -8 * (a.abs().sum() + b.abs().sum()) + 2.0 ** -17 * scale * (x.double().abs().sum(-1) * y.double().abs().amax(-1)).sum()
    assert (a.sum() - b.sum()).abs() <= bound
    for token, head, c in ((3, 1, 0), (8, 0, 17), (5, 1, 31), (6, 0, 50)):
        e = torch.zeros_like(x)
        e[token, head, c] = 1.0
        re = torch.empty_like(e)
        P.puro_rope(e, None, freq, pos, inter, re, None, scale=scale)
        terms = re.double() * y.double()  # each off by half a step
        got = float(ry[token, head, c])
        assert abs(got - float(terms.sum())) <= 2.0 ** -8 * (float(terms.abs().sum()) + abs(got)) + 2.0 ** -17 * scale * float(y[token, head].abs().max())


@pytest.mark.parametrize("rot,first,count,kind", [(128, 0, 300, "none"), (16, 2 ** 31 - 9, 9, "none"), (64, 1000003, 37, "base"), (256, 5, 1, "turns"),
                                                  (96, 131071, 65, "index")])
def test_tables(rot, first, count, kind):
    freq = P.rope_frequencies(rot, 1e4, KINDS[kind], 4.0, 8192)
    cos, sin = (torch.full((count, rot // 2), 9.0, device=DEV) for _ in range(2))
    P.puro_rope_tables(freq, first, cos, sin, scale=1.5)
    c, s = R.cos_sin(freq.cpu(), range(first, first + count), 1.5)
    for got, want in ((cos, c), (sin, s)):
        assert ((got.cpu().double() - want).abs() <= 1.5 * 2.0 ** -22 + 2.0 ** -24 * want.abs()).all()


def test_the_tables_feed_the_norms_with_a_rotation():
    """One head's rotation by the tables, through the norm with eps = 0 of rows of unit mean square, against the rotation alone."""
    t, d = 23, 64
    freq = P.rope_frequencies(d, 1e6, P.ROPE_TURNS, 4.0, 32768)
    cos, sin = torch.empty(t, d // 2, device=DEV), torch.empty(t, d // 2, device=DEV)
    P.puro_rope_tables(freq, 0, cos, sin)
    x = (torch.randint(0, 2, (t, 3, d), device=DEV) * 2 - 1).to(BF)
    a, b = torch.empty_like(x), torch.empty_like(x)
    P.puro_qk_norm_rope(x, None, None, None, 0.0, cos, sin, None, False, a, None)
    P.puro_rope(x, None, freq, None, False, b, None)
    # each within half a step and the angles' and the norm's own errors
    assert ((a.double() - b.double()).abs() <= 2.0 ** -7 * torch.maximum(a.abs(), b.abs()).double() + 2.0 ** -17).all()


def test_nothing_to_do():
    freq = P.rope_frequencies(64, 1e4)
    none = torch.empty(0, 3, 64, dtype=BF, device=DEV)
    P.puro_rope(none, None, freq, None, False, none.clone(), None)
    P.puro_rope_tables(freq, 0, torch.empty(0, 32, device=DEV), torch.empty(0, 32, device=DEV))


def test_refusals():
    freq = P.rope_frequencies(64, 1e4)
    x = torch.zeros(5, 2, 64, dtype=BF, device=DEV)
    y = torch.empty_like(x)
    with pytest.raises(ValueError):
        P.puro_rope(None, None, freq, None, False, None, None)
    with pytest.raises(ValueError):
        P.puro_rope(x.float(), None, freq, None, False, y, None)
    with pytest.raises(ValueError):
        P.puro_rope(x, None, freq, torch.zeros(4, dtype=torch.int32, device=DEV), False, y, None)
    with pytest.raises(ValueError):
        P.puro_rope(x, None, freq.cpu(), None, False, y, None)
    with pytest.raises(P.PuroError):
        P.puro_rope(x, None, P.rope_frequencies(128, 1e4), None, False, y, None)
    with pytest.raises(P.PuroError):
        P.puro_rope(x, None, freq, None, False, y[:, :1], None)
    with pytest.raises(ValueError):
        P.puro_rope_tables(freq, 0, torch.empty(4, 16, device=DEV), torch.empty(4, 16, device=DEV))


def test_on_another_stream_and_in_a_graph():
    _, q, k = qkv_views(64, 4, 2, 128)
    freq = P.rope_frequencies(128, 1e4)
    pos = torch.arange(64, dtype=torch.int32, device=DEV)
    want = [torch.empty_like(v) for v in (q, k)]
    P.puro_rope(q, k, freq, pos, False, *want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [torch.zeros_like(v) for v in (q, k)]
    side.wait_stream(torch.cuda.current_stream())
    P.puro_rope(q, k, freq, pos, False, *got, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.puro_rope(q, k, freq, pos, False, *got)
        P.puro_rope_backward(*got, freq, pos, False, *got)
    pos.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    P.puro_rope(q, k, freq, pos, False, *want)
    P.puro_rope_backward(*want, freq, pos, False, *want)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
