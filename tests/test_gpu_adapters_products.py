"""How much of a product the low-rank adapters may leave out, seen where what it is added to takes the product itself away again.

A binary32 number is the sum of three bfloat16 numbers, each the nearest to what is left: the second is at most 2^-8 of it, the third 2^-17.  Products of
second and third parts, and of thirds, are left out: of a binary32 product 2 * 2^-25 and little more, below 2^-24.  Hidden values under 16-bit
results enter as two parts, without 2^-17 of themselves.  The matrix unit adds in binary32: the largest of what it adds at a time is counted with
three roundings of 2^-24 (its own, and those of sums that differ from it by less than a factor of two)."""
import math

import pytest
import torch

import paper_2203_13483_amd as mkq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
CODE = {F32: 0, F16: 1, BF16: 2}


def _numbers(n, g, dtype=F32):
    """Numbers from 1 to 2, among them those of which a part with fewer bits leaves most, above and below."""
    x = (1.0 + torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).float()
    hard = [2.0 ** -7 - 2.0 ** -23, 2.0 ** -8 - 2.0 ** -23, 2.0 ** -8 + 2.0 ** -23, 2.0 ** -7 + 2.0 ** -14 - 2.0 ** -23, 2.0 ** -8 - 2.0 ** -17 - 2.0 ** -23,
            2.0 ** -8 - 2.0 ** -16 + 2.0 ** -17 - 2.0 ** -23, 1.0 - 2.0 ** -23]
    x[: len(hard)] = 1.0 + torch.tensor(hard, device="cuda")
    return x.to(dtype)


@pytest.mark.parametrize("M", [40, 200])
def test_hidden_values_of_binary32(M):
    g = torch.Generator("cuda").manual_seed(M)
    a, w = _numbers(M, g), _numbers(16, g)
    near = (a.double()[:, None] * w.double()).float()  # (a row takes one of the products away: a place of x for every row)
    x, down = torch.zeros(M, 8 + M, device="cuda"), torch.zeros(1, 16, 8 + M, device="cuda")
    x[:, 3], down[0, :, 3] = a, w
    x[torch.arange(M), 8 + torch.arange(M)] = 1.0
    down[0, :, 8:] = -near.T
    hidden = torch.empty(M, 16, device="cuda")
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    mkq.mkq_low_rank_adapters(x, ids, down, torch.zeros(1, 16, 8, device="cuda"), hidden=hidden)
    product = a.double()[:, None] * w.double()
    # (their places may be in different steps of a wave and in different waves: two additions more)
    assert bool(((hidden.double() - (product - near.double())).abs() <= 5 * U * product).all())


@pytest.mark.parametrize("N", [24, 300])
def test_gradients_of_binary32(N):
    """d_up = t[0] dy[0] + t[1] dy[1], with t[1] = 1 and dy[1] what takes the first product away."""
    g = torch.Generator("cuda").manual_seed(N)
    t, y = _numbers(16, g), _numbers(N, g)
    for r in range(16):
        near = (t[r].double() * y.double()).float()
        hidden = torch.zeros(2, 16, device="cuda")
        hidden[0], hidden[1] = t[r], 1.0
        down, up = torch.zeros(1, 16, 8, device="cuda"), torch.zeros(1, 16, N, device="cuda")
        dy = torch.stack([y, -near])
        _, _, d_up = mkq.mkq_low_rank_adapters_gradient(dy, torch.zeros(2, 8, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), hidden, down, up)
        product = t[r].double() * y.double()
        assert bool(((d_up[0].double() - (product - near.double())).abs() <= 4 * U * product).all()), r


@pytest.mark.parametrize("out", [F16, BF16], ids=str)
@pytest.mark.parametrize("w", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("rank", [1, 16, 40])
@pytest.mark.parametrize("M", [40, 200])
def test_results_of_16_bits(M, rank, w, out):
    g = torch.Generator("cuda").manual_seed(M + rank)
    N = 136
    x = torch.zeros(M, 8 + rank, device="cuda")
    x[:, 8:] = torch.stack([_numbers(M, g) for _ in range(rank)], 1)  # hidden values: each a value of x, times 1
    down = torch.zeros(1, rank, 8 + rank, device="cuda")
    down[0, torch.arange(rank), 8 + torch.arange(rank)] = 1.0
    up = torch.stack([_numbers(N, g, w) for _ in range(rank)])[None].contiguous()
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    hidden = torch.empty(M, rank, device="cuda")
    total = x[:, 8:].double() @ up[0].double()
    base = -total.to(out)
    got = mkq.mkq_low_rank_adapters(x, ids, down.to(w), up, None, CODE[out], base=base, hidden=hidden)
    assert torch.equal(hidden, x[:, 8:])
    want = total + base.double()
    # (sums of same-sign products: a matrix instruction for every 32 of the rank and pair of parts, the small ones first)
    tol = (2.0 ** -17 + (3 + rank / 8) * U) * total + torch.finfo(out).eps / 2 * want.abs()
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / total).max() * 2 ** 17)


@pytest.mark.parametrize("M", [40, 200])
def test_largest_and_smallest_numbers(M):
    """The largest numbers of binary32 lie above the largest of bfloat16, which is their first part; the smallest keep the bits that they have."""
    most = torch.finfo(F32).max
    x, down = torch.zeros(M, 24, device="cuda"), torch.zeros(1, 5, 24, device="cuda")
    x[0::4, 1], x[1::4, 1], x[2::4, 1], x[3::4, 1] = most, -most, 3.39e38, 1.0
    down[0, :, 1] = torch.tensor([2.0 ** -10, -(2.0 ** -126), 1.0, 0.0, 2.0 ** -20])
    x[:, 9], down[0, 3, 9] = 2.0 ** -110 * (1 + 2.0 ** -23), 2.0 ** 90
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    hidden = torch.empty(M, 5, device="cuda")
    up = torch.zeros(1, 5, 16, device="cuda")
    up[0, 2, 3], up[0, 0, 4] = 0.5, 1.0
    out = mkq.mkq_low_rank_adapters(x, ids, down, up, hidden=hidden)
    want = x.double() @ down[0].double().T.contiguous()
    assert bool(((hidden.double() - want).abs() <= 4 * U * want.abs()).all())
    assert bool(((out.double() - want @ up[0].double()).abs() <= 8 * U * (want.abs() @ up[0].double())).all())
    _, d_down, d_up = mkq.mkq_low_rank_adapters_gradient(torch.full((M, 16), most, device="cuda"), x, ids, torch.full((M, 5), 2.0 ** -9, device="cuda"), down, up)
    assert bool((d_up[0, 3] <= most).all()) and bool(((d_up.double() - M * 2.0 ** -9 * most).abs() <= 16 * U * M * 2.0 ** -9 * most).all())
    x[0, 1] = math.inf
    x[1, 1] = math.nan
    mkq.mkq_low_rank_adapters(x, ids, down, up, hidden=hidden)
    assert not hidden[0, :3].isfinite().any() and hidden[1].isnan().all() and bool(hidden[2:].isfinite().all())
