"""Activations kept in 8 bits: codes and steps bit for bit against the definition in binary64, what is made of them within counted roundings."""
import math

import pytest
import torch

import paper_2203_13483_amd as mkq

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]
CODE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available()
    mkq.load()


def _kept(x, group):
    """(codes, steps) by the definition: the step a binary32 quotient, the code decided in binary64, where a quotient of two binary32 numbers
    cannot round onto a boundary that it is not on."""
    M, K = x.shape
    groups, pitch = -(-K // group), -(-K // 32) * 32
    wide = torch.zeros(M, groups * group, dtype=torch.float32)
    wide[:, :K] = x.float().cpu()
    wide = wide.view(M, groups, group)
    fine = wide.isfinite().all(2)
    most = torch.where(fine[:, :, None], wide, 0.0).abs().amax(2)
    steps = (most.double() / 127.0).float()  # (a binary64 quotient narrowed: binary32's own quotient, for 24-bit numbers)
    steps = torch.where(most == 0, 1.0, steps.clamp(2.0 ** -126, 8454659.0 * 2.0 ** 98))  # (127 of the largest are finite)
    codes = torch.where(fine[:, :, None], wide.double() / steps.double()[:, :, None], 0.0).round().to(torch.int8).view(M, -1)
    return codes[:, :pitch].contiguous(), torch.where(fine, steps, math.nan)


def _same(a, b):
    return bool(((a == b) | ((a != a) & (b != b))).all())


def _x(M, K, dtype, seed, ld=None):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda")
    x = (x * torch.exp(torch.randn(M, 1, generator=g, device="cuda"))).to(dtype)
    if ld:
        wide = torch.full((M, ld), math.nan, device="cuda", dtype=dtype)
        wide[:, :K] = x
        x = wide[:, :K]
    return x


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,ld", [(1, 1, None), (3, 7, 9), (5, 31, None), (2, 32, None), (9, 33, 40), (4, 312, None), (37, 100, 101), (440, 768, None),
                                    (2, 1200, 1208), (3, 8193, None)])
def test_codes_steps_and_values(M, K, ld, group, dtype):
    x = _x(M, K, dtype, M + K, ld)
    codes, steps = mkq.mkq_checkpoint_int8(x, group)
    want_codes, want_steps = _kept(x, group)
    assert torch.equal(codes.cpu(), want_codes) and torch.equal(steps.cpu(), want_steps)
    value = codes[:, :K].float() * steps.repeat_interleave(group, dim=1)[:, :K]  # one rounding each, as the operator's
    for to in DTYPES:
        out = mkq.mkq_checkpoint_restore(codes, steps, K, group, CODE[to])
        assert torch.equal(out, value.to(to))
        wide = torch.full((M, K + 5), 3.0, device="cuda", dtype=to)
        mkq.mkq_checkpoint_restore(codes, steps, K, group, CODE[to], out=wide[:, :K])
        assert torch.equal(wide[:, :K], value.to(to)) and bool((wide[:, K:] == 3.0).all())


def _values(x, scale=1.0):
    """GELU and its derivative in binary64."""
    x = x.double()
    Phi = 0.5 * torch.special.erfc(-x * math.sqrt(0.5))
    return x * Phi, Phi + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("M,K,ld", [(1, 1, None), (3, 47, 49), (5, 312, None), (64, 1200, 1208), (33, 4096, None)])
def test_gelu_again_and_its_gradient(M, K, ld, dtype):
    """GELU is off by 3e-7 (its polynomial's statement) and one rounding, its derivative, of size 1.13 at most, by 4e-7 (the distribution 1e-8, two
    exponentials, three roundings of values below 1.2: 6 * 2^-24 * 1.2), and the product by two more."""
    x = _x(M, K, torch.float32, K, ld).clamp(-12, 12)
    dy = _x(M, K, dtype, K + 1, ld)
    for group in (32, 128):
        codes, steps = mkq.mkq_checkpoint_int8(x, group)
        kept = codes[:, :K].float() * steps.repeat_interleave(group, dim=1)[:, :K]
        gelu, slope = _values(kept)
        for to in {dtype, torch.float32}:
            eps = torch.finfo(to).eps / 2
            tiny = float(torch.finfo(to).smallest_normal) * eps * 2
            out = mkq.mkq_checkpoint_restore(codes, steps, K, group, CODE[to], act=mkq.MKQ_ACT_GELU).double()
            assert bool(((out - gelu).abs() <= 3e-7 + 2.0 ** -23 * gelu.abs() + eps * gelu.abs() + tiny).all())
            dx = mkq.mkq_checkpoint_gelu_gradient(codes, steps, dy, group, CODE[to]).double()
            want = dy.double() * slope
            assert bool(((dx - want).abs() <= dy.double().abs() * 4.5e-7 + (eps + 2.0 ** -23) * want.abs() + tiny).all())
        want = mkq.mkq_checkpoint_gelu_gradient(codes, steps, dy, group)
        again = dy.clone() if ld is None else torch.cat([dy, dy], 1)[:, :K]
        assert mkq.mkq_checkpoint_gelu_gradient(codes, steps, again, group, dx=again) is again
        assert torch.equal(again, want)


def test_gelu_gradient_against_differences():
    """Central differences of binary64 GELUs (step 2^-12: its third derivative, below 2, times step^2 / 6 is below 2e-8)."""
    x = torch.linspace(-9, 9, 4096, device="cuda").view(32, 128)
    codes, steps = mkq.mkq_checkpoint_int8(x, 128)
    kept = (codes.float() * steps.repeat_interleave(128, dim=1)).double()
    dx = mkq.mkq_checkpoint_gelu_gradient(codes, steps, torch.ones_like(x), 128).double()
    h = 2.0 ** -12
    slope = (_values(kept + h)[0] - _values(kept - h)[0]) / (2 * h)
    assert float((dx - slope).abs().max()) <= 5e-7


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_values_that_cannot_be_kept(dtype):
    x = _x(6, 300, dtype, 2)
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x[0, 3] = math.inf
    x[0, 70] = -math.inf
    x[1, 299] = math.nan
    x[2] = 0.0
    x[2, ::2] = -0.0
    x[3] = big
    x[3, 1] = -big
    x[4] = small
    x[4, 5] = float(small) / 4  # below the normal numbers
    x[5] = float(small) / 8
    for group in (32, 64, 128):
        codes, steps = mkq.mkq_checkpoint_int8(x, group)
        want_codes, want_steps = _kept(x, group)
        assert torch.equal(codes.cpu(), want_codes) and _same(steps.cpu(), want_steps)
        out = mkq.mkq_checkpoint_restore(codes, steps, 300, group, CODE[dtype])
        g = 3 // group
        assert out[0, : group].isnan().all() and out[1, -(300 % group):].isnan().all() and not out[2].any() and bool(out[3].isfinite().all())
        assert not out[0, -(300 % group):].isnan().any() and g == 0


def test_boundaries_are_decided_exactly():
    """Values on and beside half steps: x = (k + 1/2) step and its neighbours, for steps whose quotients are not exact."""
    rows = []
    for most in (1.0, 127.0, 3.0, 0.1, 1e-30, 1e30, 2.0 ** -120, 254.0):
        step = float((torch.tensor(most, dtype=torch.float64) / 127).float())
        half = (torch.arange(-127, 127, dtype=torch.float64) + 0.5) * step
        x = half.float()
        for v in (x, torch.nextafter(x, torch.tensor(math.inf)), torch.nextafter(x, torch.tensor(-math.inf))):
            for at in range(0, 254, 127):
                row = torch.zeros(128)
                row[:127] = v[at:at + 127]
                row[127] = most
                rows.append(row)
    x = torch.stack(rows).cuda()
    codes, steps = mkq.mkq_checkpoint_int8(x, 128)
    want_codes, want_steps = _kept(x, 128)
    assert torch.equal(codes.cpu(), want_codes) and torch.equal(steps.cpu(), want_steps)


def test_rows_past_32_bits():
    M, K = 2_200_000, 1024  # 2.25e9 codes
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    last = _x(5, K, torch.bfloat16, 3)
    x[M - 5:] = last
    codes, steps = mkq.mkq_checkpoint_int8(x, 64)
    a, b = mkq.mkq_checkpoint_int8(last, 64)
    assert torch.equal(codes[M - 5:], a) and torch.equal(steps[M - 5:], b) and not codes[M - 6].any() and bool((steps[M - 6] == 1).all())
    mkq.mkq_checkpoint_restore(codes, steps, K, 64, mkq.MKQ_BF16, out=x)
    assert torch.equal(x[M - 5:], mkq.mkq_checkpoint_restore(a, b, K, 64, mkq.MKQ_BF16))


def test_streams_and_graph_replays():
    x = _x(130, 1000, torch.float16, 1)
    dy = torch.randn(130, 1000, device="cuda")

    def run():
        codes, steps = mkq.mkq_checkpoint_int8(x, 32)
        return [codes, steps, mkq.mkq_checkpoint_restore(codes, steps, 1000, 32), mkq.mkq_checkpoint_gelu_gradient(codes, steps, dy, 32)]
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = run()
    side = torch.cuda.Stream()
    for i in range(3):
        x.copy_(_x(130, 1000, torch.float16, 10 + i))
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        side.wait_stream(torch.cuda.current_stream())
        codes, steps = mkq.mkq_checkpoint_int8(x, 32, stream=side)
        side.synchronize()
        assert torch.equal(codes, want[0]) and torch.equal(steps, want[1])
