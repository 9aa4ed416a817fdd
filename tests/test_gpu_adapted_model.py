"""A step of tuning, and answers, of adapters on a shared 4-bit model, in the calls and order of a program that does it: token rows of a 4-bit
table, kept in 8 bits for the backward pass; the shared head with every request's adapter beside it; log probabilities and their
gradient; the adapters' gradients from what was kept; clipping.  Against autograd in binary64 on the same numbers."""
import pytest
import torch

import paper_2203_13483_amd as mkq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,V,D,rank,R", [(9, 500, 64, 4, 3), (150, 2003, 312, 8, 2)])
def test_a_step_of_tuning(M, V, D, rank, R):
    g = torch.Generator("cuda").manual_seed(M)
    table = torch.randn(V, D, generator=g, device="cuda") * 0.5
    Wq, s_w = mkq.mkq_pack_weights_int4_group(table, 32)
    ids = torch.randint(0, V, (M,), generator=g, device="cuda")
    targets = torch.randint(0, V, (M,), generator=g, device="cuda")
    targets[0] = -100
    adapter = torch.randint(-1, R, (M,), generator=g, device="cuda", dtype=torch.int32)
    down = torch.randn(R, rank, D, generator=g, device="cuda") * D ** -0.5
    up = torch.randn(R, rank, V, generator=g, device="cuda") * 0.1
    scales = torch.full((R,), 2.0, device="cuda")
    weight = torch.where(targets >= 0, -1.0 / (M - 1), 0.0).float()
    bonus = torch.full((M,), -0.01 / M, device="cuda")

    x = mkq.mkq_embedding_int4_group(ids, Wq, s_w, V, D, 32)
    codes, steps = mkq.mkq_checkpoint_int8(x, 64)
    scores = mkq.mkq_linear_int4_group(x, Wq, s_w, None, V, D, 32)
    hidden = torch.empty(M, rank, device="cuda")
    mkq.mkq_low_rank_adapters(x, adapter, down, up, scales, base=scores, out=scores, hidden=hidden)
    r = mkq.mkq_token_log_probs(scores, targets, 0.8, 3)
    d_scores = mkq.mkq_token_log_probs_gradient(scores, targets, r, weight, 0.8, d_entropies=bonus)
    dx, d_down, d_up = mkq.mkq_low_rank_adapters_gradient(d_scores, codes, adapter, hidden, down, up, scales, steps=steps, group=64)
    raw = [d_down.clone(), d_up.clone()]
    norm = mkq.mkq_clip_gradients([d_down, d_up], 0.01)

    w4 = mkq.mkq_embedding_int4_group(torch.arange(V, device="cuda"), Wq, s_w, V, D, 32).double()  # the table's rows as they are
    xr, dn, u = x.double().requires_grad_(), down.double().requires_grad_(), up.double().requires_grad_()
    real, at = adapter >= 0, adapter.clamp(min=0).long()
    h = (dn[at] * xr[:, None, :]).sum(2)
    delta = torch.where(real[:, None], 2.0 * (h[:, :, None] * u[at]).sum(1), 0.0)
    z = torch.log_softmax(0.8 * (xr.detach() @ w4.T.contiguous() + delta), 1)
    lp = torch.where(targets >= 0, z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    H = -(z.exp() * z).sum(1)
    (weight.double() * lp + bonus.double() * H).sum().backward()

    def far(a, b):
        return float((a.double() - b).norm() / b.norm())
    # relative 2-norms of chains of four binary32 stages with sums of at most 2003 terms: a stage is off by less than 2003 / 5 * 2^-24 = 2.4e-5 of its
    # magnitudes; the adapters' input is read in 8 bits (half a step of 1 / 127 of the largest of 64, uniform: below 1 % of the norm)
    assert far(r.log_probs, lp.detach()) < 1e-4
    # (an entropy is the difference of two sums of the size of log V: off by an absolute 2 * 2^-24 (16 log V + V / 256 + 64) = 2.3e-5 at most and, where
    # scores are off by d, by d log V of what is not certain: a token ahead of the rest by 60 has an entropy of 1e-19)
    assert float((r.entropies.double() - H.detach()).abs().max()) < 1e-4
    assert torch.equal(r.top_tokens[:, 0].long(), scores.argmax(1))
    assert far(dx, xr.grad) < 1e-4 and far(raw[1], u.grad) < 1e-4 and far(raw[0], dn.grad) < 1e-2
    kept = mkq.mkq_checkpoint_restore(codes, steps, D, 64).double()
    # d_down is a sum of u[m] x[m]^T: with what was kept in the place of x it is exact again
    um = torch.where(real[:, None], 2.0 * (d_scores.double()[:, None, :] * up.double()[at]).sum(2), 0.0)
    want = torch.stack([um[adapter == a].T.contiguous() @ kept[adapter == a] for a in range(R)])
    assert far(raw[0], want) < 1e-4
    total = float(torch.cat([t.flatten() for t in raw]).double().norm())
    assert abs(float(norm) - total) <= 1e-6 * total and far(d_up, raw[1].double() * min(1.0, 0.01 / total)) < 1e-5


def test_answers_of_single_tokens():
    """A token each of 12 requests through a 16-bit linear whose residual is what the adapters add, GELU behind both, and the head's answers."""
    g = torch.Generator("cuda").manual_seed(3)
    M, D, V = 12, 256, 1000
    x = torch.randn(M, D, generator=g, device="cuda").half()
    W, head = torch.randn(D, D, generator=g, device="cuda") * 0.06, torch.randn(V, D, generator=g, device="cuda") * 0.1
    Wq, s_w = mkq.mkq_pack_weights_int4_group(W, 64)
    Hq, s_h = mkq.mkq_pack_weights_int4_group(head, 64)
    adapter = torch.arange(M, device="cuda", dtype=torch.int32) % 5 - 1
    down, up = (torch.randn(4, 8, D, generator=g, device="cuda").half() * 0.1 for _ in range(2))
    delta = mkq.mkq_low_rank_adapters(x, adapter, down, up)
    h = mkq.mkq_linear_int4_group(x, Wq, s_w, None, D, D, 64, act=mkq.MKQ_ACT_GELU, residual=delta)
    scores = mkq.mkq_linear_int4_group(h, Hq, s_h, None, V, D, 64, mkq.MKQ_F32)
    r = mkq.mkq_token_log_probs(scores, torch.full((M,), -100, device="cuda"), top=5)
    w4 = mkq.mkq_embedding_int4_group(torch.arange(D, device="cuda"), Wq, s_w, D, D, 64).double()
    at = adapter.clamp(min=0).long()
    t = (down[at].double() * x.double()[:, None, :]).sum(2)
    d = torch.where(adapter[:, None] >= 0, (t[:, :, None] * up[at].double()).sum(1), 0.0)
    assert float((delta.double() - d).abs().max()) <= 2.0 ** -10 * float(d.abs().max())
    y = x.double() @ w4.T.contiguous() + delta.double()
    want = y * 0.5 * torch.special.erfc(-y * 0.5 ** 0.5)
    assert float((h.double() - want).abs().max()) <= 2.0 ** -10 * float(want.abs().max())
    assert not r.log_probs.any()
    lp = torch.log_softmax(scores.double(), 1)
    assert torch.equal(r.top_tokens.long(), torch.sort(scores, dim=1, descending=True, stable=True).indices[:, :5])
    assert float((r.top_log_probs.double() - lp.gather(1, r.top_tokens.long())).abs().max()) <= 1e-5
