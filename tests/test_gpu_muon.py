"""The Muon directions against 64 bits (_muon.py)."""
import math

import pytest
import torch

import _muon as M
import paper_2608_27370_gb300 as P

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def directions(mats, steps=M.STEPS, mu=0.95, nesterov=True, stream=None, workspace=None):
    table = P.muon_table(mats)
    if workspace is None:
        workspace = torch.full((P.puro_muon_direction_workspace_size(table),), 255, dtype=torch.uint8, device=DEV)  # NaN bits
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.puro_muon_direction_grouped(table, workspace, mu, nesterov, steps, status, stream)
    return status


def check(u, v, u_type, steps=M.STEPS):
    want, bound = M.bound(v, u_type, steps)
    err = float((u.cpu().double() - want).norm())
    assert err <= bound, (err / float(want.norm()), bound / float(want.norm()))


SHAPES = [(1, 1), (1, 5), (5, 1), (1, 300), (3, 7), (8, 8), (48, 80), (64, 64), (127, 129), (129, 127), (128, 256), (256, 128), (257, 130),
          (130, 259), (300, 1000), (1000, 300), (512, 512), (515, 384), (96, 2048), (2050, 70), (255, 400), (256, 2100), (8, 32), (3000, 9),
          (32, 600), (600, 33), (20, 512), (513, 24), (320, 3000), (3, 70001), (70001, 2)]


@pytest.mark.parametrize("r,c", SHAPES)
@pytest.mark.parametrize("kind", ["mixed", "noise"])
def test_against_64_bits(r, c, kind):
    g = M.gradient(r, c, 7 * r + c, kind)
    u = torch.full((r, c), 9.0, device=DEV)
    status = directions([(g.to(DEV), None, u)])
    assert int(status) == 0
    check(u, g, F32)


@pytest.mark.parametrize("grad", [BF, F32])
@pytest.mark.parametrize("u_type", [BF, F32])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("r,c", [(72, 200), (200, 72), (33, 57)])
def test_types_and_momentum(grad, u_type, nesterov, r, c):
    g, m = M.gradient(r, c, r + c).to(grad), 3 * M.gradient(r, c, r + c + 1)
    buf, u = m.to(DEV), torch.empty(r, c, dtype=u_type, device=DEV)
    directions([(g.to(DEV), buf, u)], nesterov=nesterov, mu=0.9)
    mu = float(torch.tensor(0.9))
    want, v = M.update(g.double(), m.double(), mu, nesterov)
    assert ((buf.cpu().double() - want).abs() <= 2.0 ** -24 * want.abs()).all()  # one fused product and sum, rounded once
    check(u, v, u_type)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 6, 7])
def test_numbers_of_steps(n):
    g = M.gradient(90, 150, n, "noise")
    u = torch.empty(90, 150, device=DEV)
    steps = ((3.4445, -4.7750, 2.0315),) * n
    directions([(g.to(DEV), None, u)], steps)
    check(u, g, F32, steps)


@pytest.mark.parametrize("steps", [((1.5, -0.5, 0.0),) * 8, ((4.0, -6.0, 2.7), (3.0, -4.0, 1.8), (1.875, -1.25, 0.375)), ((0.0, 0.0, 0.0),), ((2.0, 0.0, 0.0),), ((0.25, 0.0, 0.0),) * 20,
                                   ((15 / 8, -10 / 8, 3 / 8),) * 5])
def test_other_coefficients(steps):
    g = M.gradient(70, 110, 5, "noise")
    u = torch.empty(70, 110, device=DEV)
    directions([(g.to(DEV), None, u)], steps)
    check(u, g, F32, steps)


@pytest.mark.parametrize("grad", [BF, F32])
@pytest.mark.parametrize("u_type", [BF, F32])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (2, 5), (8, 0)])
@pytest.mark.parametrize("r,c", [(40, 64), (64, 40)])
def test_views(grad, u_type, offset, pad, r, c):
    """Rows apart and starts that are not aligned: the same result, and nothing beside u is written."""
    g = M.gradient(r, c, 11).to(grad)
    wide = torch.full((r, offset + c + pad), float("nan"), dtype=grad, device=DEV)
    wide[:, offset:offset + c] = g.to(DEV)
    out = torch.full((r + 2, offset + c + pad), 5.0, dtype=u_type, device=DEV)
    u = torch.empty(r, c, dtype=u_type, device=DEV)
    directions([(g.to(DEV), None, u)])
    directions([(wide[:, offset:offset + c], None, out[1:-1, offset:offset + c])])
    assert torch.equal(out[1:-1, offset:offset + c], u)
    out[1:-1, offset:offset + c] = 5
    assert (out == 5).all()


@pytest.mark.parametrize("r,c", [(1536, 2048), (2048, 1024), (700, 8960), (4096, 2500)])
def test_signed_permutations_at_size(r, c):
    """V with one entry of each row (column) alike: all singular values are equal, and u is V times what the steps make of them; zeros stay."""
    m = min(r, c)
    g = torch.Generator().manual_seed(r)
    at = torch.randperm(max(r, c), generator=g)[:m]
    sign = (torch.randint(0, 2, (m,), generator=g) * 2 - 1).float()
    v = torch.zeros(r, c)
    if r <= c:
        v[torch.arange(m), at] = 3e-5 * sign
    else:
        v[at, torch.arange(m)] = 3e-5 * sign
    u = torch.full((r, c), 9.0, device=DEV)
    directions([(v.to(DEV), None, u)])
    want = M.singular_value(1 / math.sqrt(m)) * torch.sign(v.double())
    got = u.cpu().double()
    assert (got[v == 0] == 0).all()
    # every entry takes the same roundings, each of FP16's half step 2^-11: X, G, G's square in B, B's two products, the product with X, in
    # each of three groups: 18, of which those of the first group pass through a slope of the steps of at most 3.5 and the later of less
    assert ((got - want).abs() <= 18 * 3.5 * 2.0 ** -11 * want.abs()).all()


def test_groups_are_their_matrices():
    """More shapes and matrices than one launch takes, in any order: each direction bit for bit that of a call of its own."""
    shapes = [(8 + 5 * i % 60, 70 - 3 * i % 50) for i in range(14)] + [(32, 48)] * 130 + [(0, 5), (5, 0)] + [(300, 520), (520, 300), (1, 1)]
    mats, alone = [], []
    for i, (r, c) in enumerate(shapes):
        g = M.gradient(max(r, 1), max(c, 1), i)[:r, :c].to(DEV)
        m = M.gradient(max(r, 1), max(c, 1), 1000 + i)[:r, :c].contiguous().to(DEV) if i % 3 else None
        mats.append((g, m, torch.empty(r, c, dtype=BF if i % 2 else F32, device=DEV)))
        alone.append((g, m.clone() if m is not None else None, torch.empty_like(mats[-1][2])))
    directions(mats)
    for i in list(range(20)) + list(range(140, len(shapes))):
        directions([alone[i]])
        assert torch.equal(mats[i][2], alone[i][2]), shapes[i]
        assert mats[i][1] is None or torch.equal(mats[i][1], alone[i][1])


def test_narrow_and_wide_tiles_agree():
    """Alone its products are few tiles of 128 columns, in a group many of 256: the same sums."""
    g = [M.gradient(1100, c, c).to(DEV) for c in (1100, 2000, 1500, 1300, 1100)]
    u, alone = ([torch.empty_like(x) for x in g] for _ in range(2))
    directions([(x, None, y) for x, y in zip(g, u)])
    for x, y in zip(g, alone):
        directions([(x, None, y)])
    assert all(torch.equal(a, b) for a, b in zip(u, alone))


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 6])
@pytest.mark.parametrize("shapes", [[(48, 80), (33, 40), (700, 64), (127, 129), (256, 256), (130, 512), (65, 300)],
                                    [(20, 40), (32, 600), (5, 5), (1, 7), (400, 31), (32, 513), (16, 512), (64, 64)]])
def test_a_pair_for_each_matrix_and_launches_agree(shapes, steps):
    """Few rows, whose products one kernel takes; beside a larger matrix each product is a launch: the same sums."""
    mats = [(M.gradient(r, c, r + c).to(DEV), M.gradient(r, c, 9).to(DEV)) for r, c in shapes]
    together, beside = ([(g, m.clone(), torch.empty_like(g)) for g, m in mats] for _ in range(2))
    coefficients = (M.STEPS * 2)[:steps]
    directions(together, steps=coefficients)
    big = M.gradient(300, 320, 1).to(DEV)
    for x in beside:
        directions([x, (big, None, torch.empty_like(big))], steps=coefficients)
    for a, b, (g, m) in zip(together, beside, mats):
        assert torch.equal(a[2], b[2]), g.shape
        v = 0.95 * m.cpu() + g.cpu()
        check(a[2], g.cpu() + 0.95 * v, F32, coefficients)


@pytest.mark.parametrize("count", [77, 128])
def test_more_matrices_than_pairs(count):
    g = [M.gradient(40 + i % 2, 60, i).to(DEV) for i in range(count)]
    u = [torch.empty_like(x) for x in g]
    directions([(x, None, y) for x, y in zip(g, u)])
    for i in list(range(3)) + list(range(72, count)):
        alone = torch.empty_like(g[i])
        directions([(g[i], None, alone)])
        assert torch.equal(alone, u[i]), i


@pytest.mark.parametrize("factor", [2.0 ** -120, 2.0 ** -60, 2.0 ** 60, 2.0 ** 110])
def test_the_size_of_v_does_not_count(factor):
    g = M.gradient(50, 90, 2) * 1024
    a, b = torch.empty(50, 90, device=DEV), torch.empty(50, 90, device=DEV)
    directions([(g.to(DEV), None, a)])
    directions([((g * factor).to(DEV), None, b)])
    if factor > 2.0 ** -100:
        assert torch.equal(a, b)
    else:  # small values lose digits as FP32 numbers
        assert (a - b).norm() <= 2.0 ** -8 * a.norm()


@pytest.mark.parametrize("r,c", [(60, 200), (200, 60), (33, 71)])
@pytest.mark.parametrize("g_size,m_size", [(0.0, 1.0), (1.0, 1e5), (1e-30, 1.0), (1.0, 0.0), (1e30, 1e36), (1e-38, 1e-38)])
def test_a_gradient_that_says_nothing_of_the_momentum(r, c, g_size, m_size):
    """X is scaled by a sample of the gradient, or by the norm where that does not hold for V."""
    g, m = 1024 * M.gradient(r, c, 1) * g_size, 1024 * M.gradient(r, c, 2) * m_size
    buf, u = m.to(DEV), torch.empty(r, c, device=DEV)
    directions([(g.to(DEV), buf, u)], mu=0.5, nesterov=False)
    want, v = M.update(g.double(), m.double(), 0.5, False)
    assert ((buf.cpu().double() - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -149).all()
    check(u, buf.cpu(), F32)


@pytest.mark.parametrize("r,c", [(64, 90), (90, 64)])
def test_few_values_are_not_zero(r, c):
    g = torch.zeros(r, c)
    g[5, 7], g[40, 60], g[40, 7] = 3.0, -2.0, 1e-3
    u = torch.empty(r, c, device=DEV)
    directions([(g.to(DEV), None, u)])
    check(u, g, F32)


def test_denormal_values():
    g = M.gradient(20, 30, 9, "noise") * 2.0 ** -130
    u = torch.empty(20, 30, device=DEV)
    directions([(g.to(DEV), None, u)])
    check(u, g, F32)


def test_zero_and_what_is_not_finite():
    mats = [(torch.zeros(24, 40, device=DEV), None, torch.full((24, 40), 7.0, device=DEV))]
    for bad in (float("nan"), float("inf"), -float("inf")):
        g = M.gradient(24, 40, 4)
        g[3, 5] = bad
        mats.append((g.to(DEV), None, torch.full((24, 40), 7.0, dtype=BF, device=DEV)))
    g = M.gradient(24, 40, 4)
    mats.append((g.to(DEV), None, torch.empty(24, 40, device=DEV)))
    directions(mats)
    assert (mats[0][2] == 0).all()
    for m in mats[1:4]:
        assert torch.isnan(m[2]).all()
    check(mats[4][2], g, F32)  # beside them in the launch


def test_a_rank_of_one():
    a, b = torch.randn(60, generator=torch.Generator().manual_seed(1)), torch.randn(130, generator=torch.Generator().manual_seed(2))
    v = torch.outer(a, b)
    u = torch.empty(60, 130, device=DEV)
    directions([(v.to(DEV), None, u)])
    check(u, v, F32)


def test_twice_the_same_and_on_another_stream():
    g = M.gradient(400, 700, 1).to(DEV)
    u = [torch.empty(400, 700, device=DEV) for _ in range(3)]
    directions([(g, None, u[0])])
    directions([(g, None, u[1])])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        directions([(g, None, u[2])])
    side.synchronize()
    assert torch.equal(u[0], u[1]) and torch.equal(u[0], u[2])


@pytest.mark.parametrize("r,c", [(300, 600), (60, 100), (20, 30)])
def test_two_calls_at_once(r, c):
    """On two streams, each with its own scratch."""
    gs = [M.gradient(r, c, i).to(DEV) for i in range(2)]
    want, got = ([torch.empty(r, c, device=DEV) for _ in range(2)] for _ in range(2))
    for g, u in zip(gs, want):
        directions([(g, None, u)])
    streams = [torch.cuda.Stream() for _ in range(2)]
    table = [P.muon_table([(g, None, u)]) for g, u in zip(gs, got)]
    ws = [torch.empty(P.puro_muon_direction_workspace_size(t), dtype=torch.uint8, device=DEV) for t in table]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, w, s in zip(table, ws, streams):
            P.puro_muon_direction_grouped(t, w, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("r,c", [(130, 260), (300, 520), (24, 40)])
def test_in_a_graph(r, c):
    g, m = M.gradient(r, c, 1).to(DEV), M.gradient(r, c, 2).to(DEV)
    eager = m.clone()
    u, want = torch.empty(r, c, dtype=BF, device=DEV), torch.empty(r, c, dtype=BF, device=DEV)
    table = P.muon_table([(g, m, u)])
    ws = torch.empty(P.puro_muon_direction_workspace_size(table), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.puro_muon_direction_grouped(table, ws)
    for _ in range(3):
        graph.replay()
        directions([(g, eager, want)])
        torch.cuda.synchronize()
        assert torch.equal(u, want) and torch.equal(m, eager)
        g.mul_(-0.7)


def test_refusals():
    g = torch.zeros(8, 16, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for bad in ([(g.half(), None, g)], [(g, None, g[:, :8])], [(g, g.to(BF), g)], [(g.t(), None, g.t())], [(g[0], None, g[0])], [(g, g[:4], g)]):
        with pytest.raises(ValueError):
            P.muon_table(bad)
    with pytest.raises(P.PuroError):
        P.puro_muon_direction_grouped([(g, None, torch.empty_like(g))], ws[:1024])
    with pytest.raises(ValueError):
        P.puro_muon_direction_grouped([(g, None, torch.empty_like(g))], ws, coefficients=((1.0, 2.0),))
    with pytest.raises(P.PuroError):
        P.puro_muon_direction_grouped([(g, None, torch.empty_like(g))], ws, coefficients=())
    u, m = torch.empty_like(g), torch.zeros_like(g, dtype=F32)
    for twice in ([(g, None, u), (g, None, u)], [(g, m, u), (g, m, torch.empty_like(g))]):
        with pytest.raises(ValueError):
            P.muon_table(twice)


@pytest.mark.parametrize("r,c,count", [(1536, 2048, 1), (96, 8000, 1), (256, 1536, 70)])
def test_a_wait_that_runs_out_sets_the_status(r, c, count):
    """With no time to wait a product gives up, says so and ends; the same call then gives what it gave before.  (The waits are long: a short
    one may end before the first look at the clock.)"""
    g, u, want = M.gradient(r, c, 1).to(DEV), torch.empty(r, c, device=DEV), torch.empty(r, c, device=DEV)
    more = [(g, None, torch.empty_like(u)) for _ in range(count - 1)]
    directions([(g, None, want)] + more)
    torch.cuda.synchronize()
    P.puro_set_wait_timeout_ns(0)
    try:
        status = directions([(g, None, u)] + more)
        torch.cuda.synchronize()
    finally:
        P.puro_set_wait_timeout_ns(2_000_000_000)
    assert P.puro_fp8_get_status(status) == P.PURO_ERR_TIMEOUT
    assert P.puro_fp8_get_status(directions([(g, None, u)] + more)) == P.PURO_OK
    assert torch.equal(u, want)
