"""The Muon directions of tables of many tiles: whole models, and shapes whose tiles cannot be dealt evenly.  Each matrix's u is bit for
bit that of a call of its own, from a workspace of NaN bits."""
import pytest
import torch

import _muon as M
import paper_2608_27370_gb300 as P
from paper_2608_27370_gb300 import workloads as W
from test_gpu_muon import check, directions

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def gradient(r, c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    return (n(r, 8) @ n(8, c) / 8 ** 0.5 + 0.5 * n(r, c)) * 1e-3


def table_of(shapes, u_type):
    mats = []
    for count, r, c in shapes:
        for _ in range(count):
            mats.append((gradient(r, c, len(mats)), None, torch.full((r, c), float("nan"), dtype=u_type, device=DEV)))
    return mats


def as_alone(mats, some):
    for i in some:
        g, _, u = mats[i]
        alone = torch.empty_like(u)
        directions([(g, None, alone)])
        assert torch.equal(u, alone), (i, tuple(u.shape))


@pytest.mark.parametrize("shapes", [
    [(25, 40, 40), (1, 512, 512), (3, 384, 768), (26, 288, 2048)],
    [(2, 1024, 1664), (6, 384, 2816), (1, 256, 1152), (5, 512, 768), (3, 128, 1280), (4, 128, 2944)],
    [(10, 32, 80), (10, 3496, 874), (10, 1368, 1296)],
    [(8, 1507, 2042), (9, 1363, 4466), (8, 88, 1143)]])
def test_shapes_of_many_tiles(shapes):
    mats = table_of(shapes, F32)
    assert int(directions(mats)) == 0
    as_alone(mats, range(len(mats)))


@pytest.mark.parametrize("linears,layers", [(W.QWEN2_1P5B_LINEARS, 7), (W.QWEN2_1P5B_LINEARS, 28), (W.QWEN3_1P7B_LINEARS, 6)])
def test_whole_models(linears, layers):
    mats = table_of([(1, n, k) for _, n, k in linears] * layers, BF)
    assert int(directions(mats)) == 0
    per = len(linears)
    as_alone(mats, list(range(per)) + list(range(per * (layers // 2), per * (layers // 2 + 1))) + list(range(per * (layers - 1), per * layers)))
    assert all(bool(torch.isfinite(u).all()) for _, _, u in mats)
    g, _, u = mats[per * (layers - 2) + 1]  # (the smallest linear: 64 bits on the host)
    check(u, g.cpu(), BF)


@pytest.mark.parametrize("r,c", [(60, 200), (200, 60), (300, 520)])
def test_u_in_its_own_gradient_and_columns_of_one_matrix(r, c):
    """What may lie in the same place, or beside it in the same rows, gives what it gives apart."""
    g = [gradient(r, c, i) for i in range(3)]
    want = [torch.empty_like(x) for x in g]
    directions([(x, None, u) for x, u in zip(g, want)])
    wide = torch.cat(g, 1)
    grads, out = [wide[:, i * c:(i + 1) * c] for i in range(3)], torch.empty(r, 3 * c, device=DEV)
    directions([(x, None, out[:, i * c:(i + 1) * c]) for i, x in enumerate(grads)])
    assert all(torch.equal(out[:, i * c:(i + 1) * c], u) for i, u in enumerate(want))
    directions([(x, None, x) for x in grads])
    assert all(torch.equal(x, u) for x, u in zip(grads, want))


def test_overlaps_are_refused():
    x, u = torch.zeros(9, 40, device=DEV), torch.empty(9, 40, device=DEV)
    buf = torch.zeros(20, 40, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for bad in ([(x, x, u)], [(x, buf[:9], u), (x, buf[8:17], u.clone())], [(x, buf[:9], buf[5:14])], [(x, None, u), (x[:7], None, u[1:8])],
                [(x, None, u), (u, None, x.clone())]):
        with pytest.raises(P.PuroError):
            P.puro_muon_direction_grouped(bad, ws)
    assert (x == 0).all() and (buf == 0).all()
