"""Log probabilities, entropies and their gradient where scaled scores are far from 0, against the same formulas in binary64.

The tolerances are those of ordinary scores: an error may go by a score's distance from the row's largest, not by its size.  Only a probability
p below binary32's smallest normal number 2^-126 may count as 0, which changes scale (|d| p + |h| p (|log p| + H)) by as much as itself: at a scale of
2^28 more than the smallest number of the gradient's type, which is all that the ordinary scores' check leaves for it."""
import math

import pytest
import torch

import paper_2203_13483_amd as mkq
from test_gpu_token_log_probs import _check, _check_gradient

pytestmark = pytest.mark.gpu

LN2 = 0.693147182464599609375  # binary32's: scaled scores to the base 2 are the scores themselves, nearly


def _both(z, tokens, scale, top=5):
    r, lp, H = _check(z, tokens, scale, min(top, z.size(1)))
    assert bool(r.normalizers.isfinite().all())
    g = torch.Generator("cuda").manual_seed(z.size(1))
    d, h = torch.randn(z.size(0), generator=g, device="cuda"), torch.randn(z.size(0), generator=g, device="cuda")
    for hh in (None, h):
        grad = mkq.mkq_token_log_probs_gradient(z, tokens, r, d, scale, mkq.MKQ_F32, d_entropies=hh)
        none = lp < -126 * math.log(2.0)
        most = scale * 2.0 ** -126 * (d.double().abs()[:, None] + (0.0 if hh is None else hh.double().abs()[:, None] * (lp.abs() + H[:, None] + 1.0)))
        others = none.clone()
        others[torch.arange(z.size(0)), tokens.long()] = False
        lowest = z == -math.inf
        assert bool((grad.double().abs() <= most)[others & ~lowest].all()) and not grad[others & lowest].any()
        _check_gradient(z, tokens, scale, r, torch.where(none, -math.inf, lp), H, d, hh, torch.where(others, 0.0, grad))


@pytest.mark.parametrize("V", [3, 1000, 290000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_scores_of_any_size(V, dtype):
    g = torch.Generator("cuda").manual_seed(V)
    rows = []
    for size in (1e5, 3e6, 1e7, 1e9, 1e10, 1e15, 1e30):
        for sign in (1.0, -1.0):
            rows.append(torch.full((V,), sign * size, device="cuda"))  # all equal
            ordinary = torch.randn(V, generator=g, device="cuda")
            ordinary[V // 2] = sign * size                             # one ahead, or masked so
            rows.append(ordinary)
            rows.append(sign * size * (1.0 + torch.randint(0, 3, (V,), generator=g, device="cuda") * 2.0 ** -23))
            half = ordinary.clone()
            half[: V // 2] = -size                                     # a mask over half of the row
            rows.append(half)
    z = torch.stack(rows).to(dtype)
    tokens = torch.randint(0, V, (len(rows),), generator=g, device="cuda")
    tokens[::3] = V // 2
    _both(z, tokens, 1.0)


@pytest.mark.parametrize("V", [5, 3000, 290000])
@pytest.mark.parametrize("exponent", [-60, 12, 19, 20, 21, 23, 24, 25, 28, 31, 40, 90])
def test_scales(V, exponent):
    g = torch.Generator("cuda").manual_seed(V)
    near = 1.0 + torch.randint(0, 9, (2, V), generator=g, device="cuda") * 2.0 ** -23  # distances of the scale times 2^-23 .. 2^-20
    z = torch.cat([near, -near, torch.randn(2, V, generator=g, device="cuda"), torch.randint(0, 2, (2, V), generator=g, device="cuda").float()])
    tokens = torch.randint(0, V, (8,), generator=g, device="cuda")
    tokens[::2] = z[::2].argmax(1)
    _both(z, tokens, 2.0 ** exponent)


@pytest.mark.parametrize("V", [700, 9000, 290000])
@pytest.mark.parametrize("exponent", list(range(14, 28)))
def test_rows_around_powers_of_two(V, exponent):
    """Parts of a row, and the waves of a workgroup, whose largest scores lie on both sides of a power of two, next to each other."""
    g = torch.Generator("cuda").manual_seed(V + exponent)
    place = max(2.0 ** (exponent - 23), 2.0 ** -4)
    rows = []
    for sign in (1.0, -1.0):
        way = torch.linspace(-4.0, 4.0, V, device="cuda")
        for w in (way, way.flip(0), (way * 4).round() % 5 - 2, 8 * way):
            noise = torch.rand(V, generator=g, device="cuda")
            rows.append(sign * 2.0 ** exponent + ((w + noise) / place).round() * place)
    z = torch.stack(rows)
    tokens = torch.randint(0, V, (len(rows),), generator=g, device="cuda")
    _both(z, tokens, LN2, 20)
    some = z.clone()
    some[:, : V // 2] = -math.inf
    tokens = torch.randint(V // 2, V, (len(rows),), generator=g, device="cuda")
    _both(some, tokens, LN2, 20)


@pytest.mark.parametrize("V", [2 ** 28 + 3, 2 ** 30])
def test_the_longest_rows(V):
    z = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda")
    places = [V - 1, 0, V // 2, V - 2 ** 20, 131071, 131072 * 64, 7]
    z[0, places] = torch.tensor([12.0 - i for i in range(7)], device="cuda").bfloat16()
    tokens = torch.tensor([V - 1], device="cuda")
    r = mkq.mkq_token_log_probs(z, tokens, 1.0, 10)
    left = [p for p in range(20) if p not in places][:3]  # equal ones: the lowest tokens
    assert r.top_tokens[0].tolist() == places + left
    total = math.log(V - 7 + sum(math.exp(12.0 - i) for i in range(7)))
    want = torch.tensor([12.0 - i for i in range(7)] + [0.0] * 3, dtype=torch.float64) - total
    # (2^30 / 2^20 = 1024 terms a thread of equal powers, their joining and a logarithm: below 2^-24 (1024 + 200) of the sum)
    assert float((r.top_log_probs[0].double().cpu() - want).abs().max()) <= 2.0 ** -24 * 1300
    assert abs(float(r.log_probs[0]) - float(want[0])) <= 2.0 ** -24 * 1300
