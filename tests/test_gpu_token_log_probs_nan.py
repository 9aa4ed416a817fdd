"""Rows with NaN of any bits: their results are NaN, and their alternatives those of the other scores, a NaN as low as -infinity."""
import pytest
import torch

import paper_2203_13483_amd as mkq

pytestmark = pytest.mark.gpu

# quiet and signalling, of both signs, by what they hold
NANS = {torch.float32: (torch.int32, [0x7FC00000, 0x7F800001, 0x7FA00000, -0x400000, -0x5FFFFF, 0x7FFFFFFF]),
        torch.float16: (torch.int16, [0x7E00, 0x7C01, 0x7D00, -0x200, -0x3FF, 0x7FFF]),
        torch.bfloat16: (torch.int16, [0x7FC0, 0x7F81, 0x7FA0, -0x40, -0x7F, 0x7FFF])}


@pytest.mark.parametrize("dtype", list(NANS), ids=str)
@pytest.mark.parametrize("V,top", [(100, 5), (2100, 20), (30522, 20), (290000, 64)])
def test_alternatives_beside_nan(V, top, dtype):
    whole, bits = NANS[dtype]
    g = torch.Generator("cuda").manual_seed(V)
    rows = []
    for b in bits:
        for kind in range(5):
            z = torch.randn(V, generator=g, device="cuda").to(dtype)
            best = torch.topk(z.float(), top).indices
            at = {0: torch.randint(0, V, (1,), generator=g, device="cuda"),                      # one anywhere
                  1: torch.arange(V - 1, -1, -max(1, V // 50), device="cuda"),                   # some all over the row
                  2: (best + 1) % V, 3: (best + 6) % V,                                          # in the vectors of the largest, and in the next
                  4: torch.cat([(best + 512 * k) % V for k in range(1, 5)])}[kind]               # in the same lanes' later vectors
            n = z.view(whole).clone()
            n[at] = b
            rows.append(n)
    z = torch.stack(rows).view(dtype)
    assert bool((z != z).any(1).all())
    tokens = torch.zeros(len(rows), dtype=torch.int64, device="cuda")
    r = mkq.mkq_token_log_probs(z, tokens, 1.0, top)
    order = torch.where(z != z, -torch.inf, z.double())
    want = torch.sort(order.cpu(), dim=1, descending=True, stable=True).indices[:, :top].cuda()
    assert torch.equal(r.top_tokens.long(), want)
    assert r.log_probs.isnan().all() and r.entropies.isnan().all() and r.top_log_probs.isnan().all()
    assert torch.equal(r.normalizers[:, 0].double(), order.amax(1))
    grad = mkq.mkq_token_log_probs_gradient(z, tokens, r, torch.ones(len(rows), device="cuda"))
    assert grad.isnan().all()
