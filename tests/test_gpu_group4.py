"""The group-scaled 4-bit preparation and linear against plain implementations in 64 bits.

Tolerance of a linear: products of an activation and a code are exact, sums are binary32.  A result is K products, one scaling
per group and at most ceil(K / group) + 2 further additions away from its terms, so with S = sum |x c s| + |bias| + |residual| it is
off by at most (K + 2 groups + 4) 2^-23 S (2^-23, a whole step, for additions inside the matrix instruction, whose rounding is
not documented), plus half a step of the output's type.  GELU is off by up to 4e-7 of its own and has a slope of at most 1.13."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mkq():
    assert torch.cuda.is_available()
    import paper_2203_13483_amd as m
    m.load()
    return m


def code(m, name):
    return {"f32": m.MKQ_F32, "f16": m.MKQ_F16, "bf16": m.MKQ_BF16}[name]


def pack_codes(codes):
    """int64 codes [N, K] -> rows of nibbles with zero codes up to a multiple of 32"""
    N, K = codes.shape
    full = torch.zeros(N, -(-K // 32) * 32, dtype=torch.int64)
    full[:, :K] = codes % 16
    return (full[:, 0::2] + 16 * full[:, 1::2]).to(torch.uint8)


def weights(N, K, group, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-8, 8, (N, K), generator=g)
    s = torch.rand(N, -(-K // group), generator=g) * 0.02 + 0.001
    return codes, s


def dequantized(codes, s, group):
    return codes.double() * s.double().repeat_interleave(group, 1)[:, :codes.shape[1]]


def half_step(y, dtype):
    info = torch.finfo(dtype)
    return y.abs() * info.eps / 2 + info.smallest_normal * info.eps / 2


def reference(x, codes, s, group, bias=None, residual=None, act=False):
    """(result, S of the tolerance) in 64 bits"""
    w = dequantized(codes, s, group)
    xd = x.double()
    y, S = xd @ w.T, xd.abs() @ w.abs().T
    for more in (bias, residual):
        if more is not None:
            y, S = y + more.double(), S + more.double().abs()
    if act:
        y = y * torch.special.ndtr(y)
    return y, S


def check(got, x, codes, s, group, **kw):
    y, S = reference(x, codes, s, group, **kw)
    K = codes.shape[1]
    tol = (K + 2 * s.shape[1] + 4) * 2.0 ** -23 * S
    if kw.get("act"):
        tol = 1.13 * tol + 4e-7
    tol = tol + half_step(y.abs() + tol, got.dtype)
    off = (got.cpu().double() - y).abs()
    assert bool((off <= tol).all()), f"{float((off / tol).max())} of the tolerance at {int((off / tol).argmax())}"


SHAPES = [(1, 1, 1), (1, 5, 33), (2, 16, 32), (3, 17, 31), (16, 16, 128), (17, 40, 312), (33, 100, 257), (64, 33, 96), (70, 65, 160),
          (1, 1000, 768), (5, 130, 2049), (129, 48, 64), (128, 200, 1200), (9, 64, 4100)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(mkq, M, N, K, xt, group):
    codes, s = weights(N, K, group, M + N + K)
    g = torch.Generator().manual_seed(M * K + N)
    x = torch.randn(M, K, generator=g).to(T[xt])
    bias = torch.randn(N, generator=g)
    Wq, sd = pack_codes(codes).cuda(), s.cuda()
    for out in {xt, "f32"}:
        got = mkq.mkq_linear_int4_group(x.cuda(), Wq, sd, bias.cuda(), N, K, group, code(mkq, out))
        assert got.dtype == T[out]
        check(got, x, codes, s, group, bias=bias)
    check(mkq.mkq_linear_int4_group(x.cuda(), Wq, sd, None, N, K, group, mkq.MKQ_F32), x, codes, s, group)


@pytest.mark.parametrize("xt,out,rt", [("f16", "f16", "f16"), ("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f16", "f32", "bf16"), ("f32", "bf16", "f16")])
@pytest.mark.parametrize("M,N,K", [(1, 37, 312), (20, 70, 96), (100, 130, 200)])
def test_epilogue(mkq, M, N, K, xt, out, rt):
    codes, s = weights(N, K, 64, 5)
    g = torch.Generator().manual_seed(6)
    x, bias = torch.randn(M, K, generator=g).to(T[xt]), torch.randn(N, generator=g)
    residual = torch.randn(M, N, generator=g).to(T[rt])
    Wq, sd = pack_codes(codes).cuda(), s.cuda()
    got = mkq.mkq_linear_int4_group(x.cuda(), Wq, sd, bias.cuda(), N, K, 64, code(mkq, out), act=mkq.MKQ_ACT_GELU, residual=residual.cuda())
    check(got, x, codes, s, 64, bias=bias, residual=residual, act=True)
    got = mkq.mkq_linear_int4_group(x.cuda(), Wq, sd, None, N, K, 64, code(mkq, out), residual=residual.cuda())
    check(got, x, codes, s, 64, residual=residual)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [1, 4, 16, 40, 128, 200])
def test_whole_numbers_are_exact(mkq, M, xt, group):
    """Whole activations, steps that are powers of two: every sum is exact, so is every result (which also names each place
    of a code: a pair of operands in another order would not give these sums)."""
    N, K = 70, 1000
    g = torch.Generator().manual_seed(M + group)
    codes = torch.randint(-8, 8, (N, K), generator=g)
    s = 2.0 ** torch.randint(-3, 4, (N, -(-K // group)), generator=g).float()
    x = torch.randint(-15, 16, (M, K), generator=g).to(T[xt])
    got = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, N, K, group, mkq.MKQ_F32)
    assert torch.equal(got.cpu().double(), x.double() @ dequantized(codes, s, group).T)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(3, 20003, 136), (5, 25700, 264), (16, 13001, 1030), (20, 26001, 392), (45, 26001, 160), (100, 25999, 520), (128, 3205, 2056), (130, 3250, 4100),
                                   (16, 40, 4360), (7, 6500, 2056), (2, 6401, 8200), (9, 25601, 300), (64, 4000, 1240)])
def test_every_tile_is_exact_on_whole_numbers(mkq, M, N, K, xt, group):
    """As above where the grid is large enough for tiles of 32 and 64 tokens and for waves that share nothing, with K that ends
    within a chunk, within a step and within a piece"""
    g = torch.Generator("cuda").manual_seed(M + N + K)
    codes = torch.randint(-8, 8, (N, -(-K // 32) * 32), generator=g, device="cuda")
    codes[:, K:] = 0
    s = 2.0 ** torch.randint(-3, 4, (N, -(-K // group)), generator=g, device="cuda").float()
    x = torch.randint(-15, 16, (M, K), generator=g, device="cuda").to(T[xt])
    Wq = ((codes[:, 0::2] % 16) + 16 * (codes[:, 1::2] % 16)).to(torch.uint8)
    got = mkq.mkq_linear_int4_group(x, Wq, s, None, N, K, group, mkq.MKQ_F32)
    w = codes[:, :K].double() * s.double().repeat_interleave(group, 1)[:, :K]
    assert torch.equal(got.double(), x.double() @ w.T.contiguous())


@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [3, 50])
@pytest.mark.parametrize("pad", [8, 3])
def test_rows_with_gaps(mkq, xt, M, pad):
    """x with a row stride, aligned and not; what lies between its rows is NaN and must not be read into the result"""
    N, K, group = 50, 313, 32
    codes, s = weights(N, K, group, 1)
    wide = torch.full((M, K + 7 + pad), float("nan")).to(T[xt])
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).to(T[xt])
    wide[:, :K] = x
    got = mkq.mkq_linear_int4_group(wide.cuda()[:, :K], pack_codes(codes).cuda(), s.cuda(), None, N, K, group, mkq.MKQ_F32)
    check(got, x, codes, s, group)


@pytest.mark.parametrize("M", [6, 70])
def test_infinities_and_nan_stay_in_their_rows(mkq, M):
    N, K, group = 40, 200, 64
    codes, s = weights(N, K, group, 3)
    codes[:, 7] = torch.where(codes[:, 7] == 0, 1, codes[:, 7])
    codes[5, 7] = 0
    for xt in T:
        x = torch.randn(M, K, generator=torch.Generator().manual_seed(4)).to(T[xt])
        clean = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, N, K, group, mkq.MKQ_F32).cpu()
        x[1, 7], x[3, 7] = float("inf"), float("nan")
        got = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, N, K, group, mkq.MKQ_F32).cpu()
        rows = [m for m in range(M) if m not in (1, 3)]
        assert torch.equal(got[rows], clean[rows])
        assert bool(got[3].isnan().all())
        sign = codes[:, 7].sign().float()
        want = torch.where(sign == 0, float("nan"), sign * float("inf"))
        assert torch.equal(got[1].isnan(), want.isnan()) and torch.equal(got[1][~want.isnan()], want[~want.isnan()])


def test_a_nan_whose_payload_is_low_stays_one(mkq):
    codes, s = weights(16, 32, 32, 8)
    x = torch.zeros(1, 32)
    x.view(torch.int32)[0, 3] = 0x7F800001
    got = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, 16, 32, 32, mkq.MKQ_F32)
    assert bool(got.isnan().all())


def test_large_and_small_activations(mkq):
    """binary32 near both ends of its range, binary16 below its normal numbers: one activation a row, so only roundings of the
    product with the step are left (whole powers of two: none)"""
    N = 16
    codes = torch.arange(-8, 8).reshape(N, 1)
    s = torch.ones(N, 1)
    for xt, values in (("f32", [3.0e37, 1.2345678e-30, 1.9999999, 16777215.0, 2.0 ** -100 * 8388609]), ("f16", [2.0 ** -24, 3 * 2.0 ** -24, 1023 * 2.0 ** -24, 65504.0]),
                       ("bf16", [1.0e37, 1.0e-30])):
        x = torch.tensor(values).reshape(-1, 1).to(T[xt])
        got = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, N, 1, 32, mkq.MKQ_F32).cpu()
        exact = x.double() @ codes.double().T
        # a product of 24 bits and 4 has up to 27: one rounding, in three parts two
        assert bool(((got.double() - exact).abs() <= 2.0 ** -23 * exact.abs()).all()), (xt, got, exact)
        if xt != "f32":
            assert torch.equal(got.double(), exact)


@pytest.mark.parametrize("M,N,K,xt", [(1, 30522, 768, "f16"), (16, 28672, 2048, "bf16"), (128, 5000, 1024, "f16"), (3, 7, 28672, "f32")])
def test_large(mkq, M, N, K, xt):
    """Sampled channels of large calls; the whole of the result is written, nothing behind it"""
    group = 128
    g = torch.Generator("cuda").manual_seed(1)
    Wq = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = torch.rand(N, K // group, device="cuda", generator=g) * 0.02
    x = torch.randn(M, K, device="cuda", generator=g).to(T[xt])
    room = torch.full((M * N + 64,), -77.0, device="cuda", dtype=torch.float32)
    got = mkq.mkq_linear_int4_group(x, Wq, s, None, N, K, group, mkq.MKQ_F32, out=room[:M * N].view(M, N))
    assert bool((room[M * N:] == -77.0).all()) and bool((got != -77.0).all())
    rows = torch.cat([torch.arange(min(N, 40)), torch.randint(0, N, (40,)), torch.arange(max(0, N - 40), N)])
    b = Wq[rows.cuda()].cpu().long()
    codes = torch.stack((b % 16, b // 16), -1).flatten(1)
    codes = torch.where(codes > 7, codes - 16, codes)
    check(got[:, rows.cuda()], x.cpu(), codes, s[rows.cuda()].cpu(), group)


def test_weights_past_32_bits(mkq):
    """More than 2^32 bytes of weights: the first and last channels, exact on whole numbers"""
    N, K, group = 70000, 131072, 128
    g = torch.Generator("cuda").manual_seed(3)
    Wq = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = 2.0 ** torch.randint(-2, 2, (N, K // group), device="cuda", generator=g).float()
    x = torch.randint(-3, 4, (2, K), device="cuda", generator=g).half()
    got = mkq.mkq_linear_int4_group(x, Wq, s, None, N, K, group, mkq.MKQ_F32)
    rows = torch.tensor([0, 1, 32767, 32768, 65535, 65536, 69999], device="cuda")
    b = Wq[rows].long()
    codes = torch.stack((b % 16, b // 16), -1).flatten(1)
    w = torch.where(codes > 7, codes - 16, codes).double() * s[rows].double().repeat_interleave(group, 1)
    assert torch.equal(got[:, rows].double(), x.double() @ w.T.contiguous())


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("wt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,K", [(1, 1), (5, 31), (7, 312), (3, 2049), (40, 768), (2, 5000)])
def test_pack(mkq, N, K, wt, group):
    g = torch.Generator().manual_seed(N + K)
    W = (torch.randn(N, K + 5, generator=g) * 0.05).to(T[wt])
    W[:, ::7] *= 3
    W[0, :40] = 0
    for lo, hi in ((0, K), (0, K)):
        Wv = W[:, lo:hi] if K % 2 else W[:, lo:hi].contiguous()
        Wq, s = mkq.mkq_pack_weights_int4_group(Wv.cuda() if K % 2 == 0 else W.cuda()[:, lo:hi], group)
        groups = -(-K // group)
        padded = torch.zeros(N, groups * group)
        padded[:, :K] = Wv.float()
        mx = padded.view(N, groups, group).abs().amax(-1)
        want = torch.where(mx > 0, mx / np.float32(7), torch.ones_like(mx))
        assert torch.equal(s.cpu(), want)
        q = (padded.view(N, groups, group) / want[..., None]).clamp(-8, 7).round().view(N, -1)[:, :K].long()
        assert torch.equal(Wq.cpu(), pack_codes(q))
    given = torch.rand(N, groups, generator=g) * 0.05 + 0.005
    Wq, s = mkq.mkq_pack_weights_int4_group(Wv.contiguous().cuda(), group, given.cuda())
    assert torch.equal(s.cpu(), given)
    q = (padded.view(N, groups, group) / given[..., None]).clamp(-8, 7).round().view(N, -1)[:, :K].long()
    assert torch.equal(Wq.cpu(), pack_codes(q))


def test_pack_of_nan_and_infinity(mkq):
    W = torch.randn(2, 64)
    W[0, 3], W[1, 40] = float("nan"), float("inf")
    Wq, s = mkq.mkq_pack_weights_int4_group(W.cuda(), 32)
    s = s.cpu()
    assert bool(torch.isfinite(s[0]).all()) and math.isinf(float(s[1, 1])) and math.isfinite(float(s[1, 0]))
    nib = Wq.cpu().long()
    codes = torch.stack((nib % 16, nib // 16), -1).flatten(1)
    assert int(codes[0, 3]) == 0 and int(codes[1, 32:].abs().sum()) == 0  # NaN -> 0; finite / inf = 0, inf / inf = NaN -> 0


def test_empty_and_other_stream(mkq):
    N, K = 64, 256
    codes, s = weights(N, K, 64, 9)
    Wq, sd = pack_codes(codes).cuda(), s.cuda()
    assert mkq.mkq_linear_int4_group(torch.zeros(0, K, device="cuda"), Wq, sd, None, N, K).shape == (0, N)
    x = torch.randn(5, K)
    side = torch.cuda.Stream()
    xd = x.cuda()
    side.wait_stream(torch.cuda.current_stream())
    got = mkq.mkq_linear_int4_group(xd, Wq, sd, None, N, K, 64, stream=side)
    side.synchronize()
    check(got, x, codes, s, 64)


def test_captured(mkq):
    N, K, M = 200, 320, 40
    codes, s = weights(N, K, 32, 10)
    Wq, sd = pack_codes(codes).cuda(), s.cuda()
    x, out = torch.zeros(M, K, device="cuda", dtype=torch.float16), torch.empty(M, N, device="cuda", dtype=torch.float16)
    run = lambda: mkq.mkq_linear_int4_group(x, Wq, sd, None, N, K, 32, mkq.MKQ_F16, out=out)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        x.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(i)))
        run()
        want = out.clone()
        out.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("M", [6, 70])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
def test_gelu_of_infinities_and_nan(mkq, M, out):
    """GELU is x Phi(x): +infinity stays one, -infinity times 0 is a NaN as in IEEE arithmetic, a NaN stays one"""
    N, K, group = 40, 200, 64
    codes, s = weights(N, K, group, 3)
    codes[:, 7] = torch.where(codes[:, 7] == 0, 1, codes[:, 7])
    sign = codes[:, 7].sign().float()
    Wq, sd = pack_codes(codes).cuda(), s.cuda()
    for xt in T:
        x = torch.randn(M, K, generator=torch.Generator().manual_seed(4)).to(T[xt])
        run = lambda x, **kw: mkq.mkq_linear_int4_group(x.cuda(), Wq, sd, kw.pop("bias", None), N, K, group, code(mkq, out), act=mkq.MKQ_ACT_GELU, **kw).cpu()
        clean = run(x)
        x[1, 7], x[2, 7], x[3, 7] = float("inf"), float("-inf"), float("nan")
        got = run(x)
        rows = [m for m in range(M) if m not in (1, 2, 3)]
        assert torch.equal(got[rows], clean[rows]) and bool(got[3].isnan().all())
        for row, up in ((1, sign > 0), (2, sign < 0)):
            assert bool((got[row][up] == math.inf).all()) and bool(got[row][~up].isnan().all())
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(4))
    clean = run(x)
    bias, residual = torch.zeros(N), torch.zeros(M, N)
    bias[3], residual[2, 5] = float("inf"), float("inf")
    got = run(x, bias=bias.cuda(), residual=residual.cuda())
    assert bool((got[:, 3] == math.inf).all()) and float(got[2, 5]) == math.inf
    got[:, 3], got[2, 5] = clean[:, 3], clean[2, 5]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("M,N", [(3, 40), (50, 6000)])
def test_binary32_activations_down_to_the_smallest(mkq, M, N):
    """Three bfloat16 parts hold what is a multiple of 2^-133, all 24 bits from 2^-110 up: a smaller activation is off by less than
    2^-133, and the sum of K products, which steps of 1 leave alone, by K 2^-23 of their sizes and half a step of 2^-149 each."""
    K = 40
    g = torch.Generator().manual_seed(M)
    codes = torch.randint(-8, 8, (N, K), generator=g)
    s = torch.ones(N, 2)
    for low, high in ((-149, -140), (-140, -126), (-126, -118), (-118, -110), (-110, -100)):
        x = torch.ldexp(torch.rand(M, K, generator=g, dtype=torch.float64) + 0.5, torch.randint(low, high, (M, K), generator=g)).float()
        got = mkq.mkq_linear_int4_group(x.cuda(), pack_codes(codes).cuda(), s.cuda(), None, N, K, 32, mkq.MKQ_F32).cpu()
        xd, c = x.double(), codes.double()
        S = xd @ c.abs().T
        lost = (xd < 2.0 ** -110).double() * 2.0 ** -133 @ c.abs().T
        tol = lost + (3 * K + 4) * 2.0 ** -23 * (S + lost) + (3 * K + 4) * 2.0 ** -149
        off = (got.double() - xd @ c.T).abs()
        assert bool((off <= tol).all()), (low, float((off / tol).max()))


@pytest.mark.parametrize("xt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1030, 333, 264), (4097, 40, 96), (515, 5000, 520)])
def test_many_tokens_are_exact_on_whole_numbers(mkq, M, N, K, xt):
    """Scores of every position of a batch: many tiles of tokens, the last one short"""
    g = torch.Generator("cuda").manual_seed(M)
    codes = torch.randint(-8, 8, (N, -(-K // 32) * 32), generator=g, device="cuda")
    codes[:, K:] = 0
    s = 2.0 ** torch.randint(-3, 4, (N, -(-K // 64)), generator=g, device="cuda").float()
    x = torch.randint(-15, 16, (M, K), generator=g, device="cuda").to(T[xt])
    Wq = ((codes[:, 0::2] % 16) + 16 * (codes[:, 1::2] % 16)).to(torch.uint8)
    room = torch.full((M * N + 64,), -77.25, device="cuda")
    got = mkq.mkq_linear_int4_group(x, Wq, s, None, N, K, 64, mkq.MKQ_F32, out=room[:M * N].view(M, N))
    w = codes[:, :K].double() * s.double().repeat_interleave(64, 1)[:, :K]
    assert torch.equal(got.double(), x.double() @ w.T.contiguous()) and bool((room[M * N:] == -77.25).all())
