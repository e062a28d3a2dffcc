"""The bound on the Muon kernels' waits counts their own work, not the kernel before them: the one that writes X once more, where the
gradient said nothing of the momentum, takes more than ten microseconds on a few SMs while the products' blocks are there already."""
import pytest
import torch

import paper_2608_27370_gb300 as P
from test_gpu_muon_tables import gradient

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("count,r,c", [(1, 512, 512), (1, 2048, 640), (24, 128, 1536), (12, 1536, 128)])
def test_a_short_bound_is_not_used_up_by_the_kernel_before(count, r, c):
    mats = [(gradient(r, c, i), 1e5 * gradient(r, c, 100 + i), torch.empty(r, c, device=DEV)) for i in range(count)]
    table = P.muon_table(mats)
    ws = torch.empty(P.puro_muon_direction_workspace_size(table), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.puro_muon_direction_grouped(table, ws, 1.0, False, dev_status=status)
    torch.cuda.synchronize()
    P.puro_set_wait_timeout_ns(6000)
    try:
        for _ in range(5):
            P.puro_muon_direction_grouped(table, ws, 1.0, False, dev_status=status)
            torch.cuda.synchronize()
    finally:
        P.puro_set_wait_timeout_ns(2_000_000_000)
    assert int(status) == P.PURO_OK
