"""Calls of the low-rank adapters that lie at the edges of what they allow, against the same formulas in binary64."""
import pytest
import torch

import paper_2203_13483_amd as mkq
from test_gpu_adapters import CODE, Case, _near

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("M,K,N", [(16, 768, 768), (64, 1024, 1024), (65, 768, 768), (300, 200, 328)])
def test_results_beside_their_rows(M, K, N):
    """x and out as columns of one wide matrix; over each other they are refused, whatever the sizes."""
    c = Case(M, K, N, 8, 5, F16, F16, F16, "mixed")
    wide = torch.full((M, K + N + 8), 3.0, dtype=F16, device="cuda")
    x, out = wide[:, :K], wide[:, K + 8:]  # (a multiple of 16 bytes on)
    x.copy_(c.x)
    out.copy_(c.base)
    mkq.mkq_low_rank_adapters(x, c.ids, c.down, c.up, c.scales, base=out, out=out)
    _, _, y, tol = c.forward(c.base)
    _near(out, y, tol, "out")
    assert torch.equal(x, c.x) and bool((wide[:, K:K + 8] == 3.0).all())
    again = wide[:, 8:8 + N]
    for base in (None, again):
        with pytest.raises(mkq.MkqError):
            mkq.mkq_low_rank_adapters(x, c.ids, c.down, c.up, c.scales, base=base, out=again)
    assert torch.equal(x, c.x)
