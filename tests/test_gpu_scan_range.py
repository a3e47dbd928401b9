"""The scan at the ends of float's range."""
import pytest
import torch

from ops_common import dev, rng
from seq_common import on_gpu, packed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,n", [(1, 1), (5, 3), (70, 16), (1, 17), (70, 40)])
def test_an_infinite_B_makes_dC_infinite(d, n):
    """B of one state is infinite in the third event: from there on that state is, and its dC, a sum of positive multiples of it over columns
    that do not fill a wavefront.  Nothing else of dC changes."""
    from paper_2307_07649_amd import tgnn
    q, g = packed([9]), rng(d + n)
    t = dict(x=dev(g.uniform(0.5, 1.5, (9, d)), torch.float32), dt=dev(g.uniform(-1, 1, (9, d)), torch.float32),
             B=dev(g.uniform(0.5, 1.5, (9, n)), torch.float32), C=dev(g.uniform(0.5, 1.5, (9, n)), torch.float32),
             A=dev(-g.uniform(0.2, 1.0, (d, n)), torch.float32))
    dy = dev(g.uniform(0.5, 1.5, (9, d)), torch.float32)
    clean = tgnn.tgnn_selective_scan_bwd(on_gpu(tgnn, q), dy, **t)["dC"].clone()
    t["B"][2, n - 1] = float("inf")
    got = tgnn.tgnn_selective_scan_bwd(on_gpu(tgnn, q), dy, **t)["dC"]
    assert (got[2:, n - 1] == float("inf")).all()
    got[2:, n - 1] = clean[2:, n - 1]
    assert torch.equal(got, clean)
