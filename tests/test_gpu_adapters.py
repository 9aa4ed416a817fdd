"""Low-rank adapters and their gradients against the same formulas in binary64.

Tolerances: products are exact, and a sum of n of them passes through at most n / 32 additions of each of up to six parts and 64 more (inside
the matrix unit, across waves, across splits): u (n / 5 + 64) of the sum of their magnitudes, u = 2^-24.  What is computed from a hidden value has
its error times the factor, results of 16 bits may leave out 2^-16 of a product, and a result is rounded once to its type."""
import pytest
import torch

import paper_2203_13483_amd as mkq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
CODE = {F32: 0, F16: 1, BF16: 2}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available()
    mkq.load()


def _ids(M, R, order, g):
    if order == "requests":  # ragged, one after the other, some without an adapter
        n = max(1, M // 7)
        cuts = torch.randint(0, M, (n - 1,), generator=g, device="cuda").sort().values
        ids = torch.randint(-1, R, (n,), generator=g, device="cuda")
        ids = ids[torch.bucketize(torch.arange(M, device="cuda"), cuts, right=True)]
    elif order == "mixed":
        ids = torch.randint(-1, R, (M,), generator=g, device="cuda")
    elif order == "strange":
        ids = torch.tensor([R, -5, 2 ** 31 - 1, -2 ** 31, 0, R - 1], device="cuda")[torch.randint(0, 6, (M,), generator=g, device="cuda")]
    elif order == "none":
        ids = torch.full((M,), -1, device="cuda")
    else:
        ids = torch.full((M,), R - 1, device="cuda")
    return ids.to(torch.int32)


def _rows(M, K, dtype, g, gap=0):
    x = torch.randn(M, K, generator=g, device="cuda").to(dtype)
    if gap:
        wide = torch.full((M, K + gap), float("nan"), device="cuda", dtype=dtype)
        wide[:, :K] = x
        x = wide[:, :K]
    return x


class Case:
    def __init__(self, M, K, N, rank, R, x, w, out, order, seed=0, gap=0):
        g = torch.Generator("cuda").manual_seed(seed + M + K + N + rank)
        self.M, self.K, self.N, self.rank, self.R, self.out = M, K, N, rank, R, out
        self.ids = _ids(M, R, order, g)
        self.x, self.dy = _rows(M, K, x, g, gap), _rows(M, N, out, g, gap)
        self.down = (torch.randn(R, rank, K, generator=g, device="cuda") * K ** -0.5).to(w)
        self.up = (torch.randn(R, rank, N, generator=g, device="cuda") * 0.3).to(w)
        self.scales = torch.rand(R, generator=g, device="cuda") + 0.5
        self.base, self.dx_base = _rows(M, N, out, g, gap), _rows(M, K, out, g)
        self.real = (self.ids >= 0) & (self.ids < R)
        self.at = torch.where(self.real, self.ids, 0).long()

    def _own(self, w, x):
        """w_a x for every row's own adapter, and the same of magnitudes: [M, rank]."""
        t = torch.zeros(self.M, self.rank, dtype=torch.float64, device="cuda")
        s = torch.zeros_like(t)
        for a in range(self.R):
            rows = torch.nonzero(self.real & (self.ids == a)).flatten()
            wa = w[a].double().T.contiguous()
            t[rows], s[rows] = x[rows].double() @ wa, x[rows].double().abs() @ wa.abs()
        return t, s

    def _spread(self, t, w, n):
        y = torch.zeros(self.M, n, dtype=torch.float64, device="cuda")
        for a in range(self.R):
            rows = torch.nonzero(self.real & (self.ids == a)).flatten()
            y[rows] = t[rows] @ w[a].double()
        return y

    def forward(self, base, scales=True):
        """(hidden, its tolerance, out, its tolerance)"""
        s = (self.scales if scales else torch.ones_like(self.scales))[self.at].double()[:, None]
        t, size = self._own(self.down, self.x)
        t_tol = U * (self.K / 5 + 64) * size
        y = s * self._spread(t, self.up, self.N)
        wabs = self.up.double().abs()
        spread = s * self._spread(t.abs(), wabs, self.N)
        tol = s * self._spread(t_tol, wabs, self.N) + spread * (U * (self.rank / 5 + 64) + (0 if self.out == F32 else 2.0 ** -16))
        if base is not None:
            y = y + base.double()
        tol = tol + (torch.finfo(self.out).eps / 2 + 2 * U) * (y.abs() + tol) + 2.0 ** -25
        return t, t_tol, y, tol

    def backward(self, hidden, x, base):
        """dx, d_down, d_up with their tolerances, from the hidden values that the forward pass gave"""
        s = self.scales[self.at].double()[:, None]
        u, size = self._own(self.up, self.dy)
        u, u_tol = s * u, s * U * (self.N / 5 + 66) * size
        dabs = self.down.double().abs()
        dx = self._spread(u, self.down, self.K)
        tol = self._spread(u_tol, dabs, self.K) + self._spread(u.abs(), dabs, self.K) * (U * (self.rank / 5 + 64) + (0 if self.out == F32 else 2.0 ** -16))
        if base is not None:
            dx = dx + base.double()
        got = [(dx, tol + (torch.finfo(self.out).eps / 2 + 2 * U) * (dx.abs() + tol) + 2.0 ** -25)]
        for c, c_tol, y, f in ((u, u_tol, x.double(), None), (hidden.double(), torch.zeros_like(u), self.dy.double(), self.scales.double())):
            grad = torch.zeros(self.R, self.rank, y.size(1), dtype=torch.float64, device="cuda")
            g_tol = torch.zeros_like(grad)
            for a in range(self.R):
                rows = torch.nonzero(self.real & (self.ids == a)).flatten()
                ct, yr = c[rows].T.contiguous(), y[rows]
                grad[a] = ct @ yr
                g_tol[a] = c_tol[rows].T.contiguous() @ yr.abs() + U * (len(rows) / 5 + 66) * (ct.abs() @ yr.abs())
                if f is not None:
                    grad[a] *= f[a]
                    g_tol[a] *= f[a]
            got.append((grad, g_tol))
        return got


def _near(got, want, tol, what):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (what, float(err.max()), float((err / tol.clamp(min=1e-300)).max()))


def _check(c, gap=0):
    M, K, N = c.M, c.K, c.N
    hidden = torch.full((M, c.rank), float("nan"), device="cuda")
    t, t_tol, y, tol = c.forward(c.base)
    out = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, CODE[c.out], base=c.base, hidden=hidden)
    _near(hidden, t, t_tol, "hidden")
    _near(out, y, tol, "out")
    if not c.real.all():
        assert torch.equal(out[~c.real], c.base[~c.real]) and not hidden[~c.real].any()
    _, _, y, tol = c.forward(None, scales=False)
    bare = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, None, CODE[c.out])
    _near(bare, y, tol, "out without base and scales")
    wide = torch.full((M, N + 5), 9.0, device="cuda", dtype=c.out)
    wide[:, :N] = c.base
    mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, CODE[c.out], base=wide[:, :N], out=wide[:, :N])
    assert torch.equal(wide[:, :N], out) and bool((wide[:, N:] == 9.0).all())
    _check_gradient(c, hidden)


def _check_gradient(c, hidden):
    for grad in {F32, c.down.dtype}:
        got = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales, CODE[c.out], CODE[grad], base=c.dx_base)
        for g, (want, tol), what in zip(got, c.backward(hidden, c.x, c.dx_base), ("dx", "d_down", "d_up")):
            if what != "dx":
                tol = tol + (torch.finfo(grad).eps / 2) * (want.abs() + tol) + 2.0 ** -25
            _near(g, want, tol, what)
    again = [torch.full_like(t, 0.5) for t in got[1:]]
    dx, _, _ = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales, CODE[c.out], CODE[grad], base=c.dx_base,
                                                  d_down=again[0], d_up=again[1], accumulate=True)
    assert torch.equal(dx, got[0])
    empty = torch.bincount(c.at[c.real], minlength=c.R) == 0
    for t, g in zip(again, got[1:]):
        assert bool((t[empty] == 0.5).all()) and not g[empty].any()
        eps = torch.finfo(grad).eps
        assert bool(((t.double() - g.double() - 0.5).abs() <= eps * (g.double().abs() + 0.5)).all())
    none, d_down, d_up = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales, CODE[c.out], CODE[grad], want_dx=False)
    # (without dx the places of a row are not split: other partial sums)
    _near(d_down, c.backward(hidden, c.x, None)[1][0], c.backward(hidden, c.x, None)[1][1] + torch.finfo(grad).eps * d_down.double().abs() + 2.0 ** -24, "d_down alone")
    assert none is None and torch.equal(d_up, got[2])


SIZES = [(1, 24, 24, 1, 1), (1, 768, 768, 8, 3), (2, 33, 40, 3, 2), (15, 100, 65, 4, 40), (16, 768, 1024, 16, 16), (17, 312, 1200, 16, 2),
         (64, 1000, 129, 17, 5), (65, 64, 128, 32, 64), (130, 257, 515, 33, 7), (437, 312, 1200, 4, 1), (513, 130, 130, 64, 3),
         (600, 96, 72, 65, 2), (40, 48, 40, 256, 2), (2100, 72, 136, 8, 4), (3000, 40, 24, 16, 300)]


@pytest.mark.parametrize("types", [(F16, F16, F16), (BF16, BF16, BF16), (F32, F32, F32)], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("order", ["requests", "mixed", "one"])
@pytest.mark.parametrize("M,K,N,rank,R", SIZES)
def test_against_binary64(M, K, N, rank, R, order, types):
    _check(Case(M, K, N, rank, R, *types, order, gap=3 if M % 2 else 0))


@pytest.mark.parametrize("x", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("w", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("out", [F32, F16, BF16], ids=str)
def test_types(x, w, out):
    _check(Case(70, 200, 136, 12, 3, x, w, out, "requests"))


@pytest.mark.parametrize("order", ["strange", "none"])
@pytest.mark.parametrize("M", [3, 100, 2500])
def test_rows_without_an_adapter(M, order):
    _check(Case(M, 72, 80, 8, 5, BF16, BF16, BF16, order))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(5, 33), (130, 312), (700, 1030)])
def test_gradient_from_a_checkpoint(M, K, group):
    c = Case(M, K, 96, 9, 3, BF16, BF16, F32, "requests")
    hidden = torch.randn(M, 9, device="cuda") * c.real[:, None]
    codes, steps = mkq.mkq_checkpoint_int8(c.x, group)
    kept = mkq.mkq_checkpoint_restore(codes, steps, K, group)
    got = mkq.mkq_low_rank_adapters_gradient(c.dy, codes, c.ids, hidden, c.down, c.up, c.scales, steps=steps, group=group)
    for g, (want, tol), what in zip(got, c.backward(hidden, kept, None), ("dx", "d_down", "d_up")):
        _near(g, want, tol + 2.0 ** -25, what)


def test_infinities_and_nan_stay_where_they_belong():
    nan, inf = float("nan"), float("inf")
    for M in (40, 600, 2200):
        for w in (F16, BF16, F32):
            c = Case(M, 72, 80, 12, 4, w, w, w, "mixed")
            clean = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base)
            hidden = torch.empty(M, 12, device="cuda")
            mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, hidden=hidden)
            want = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales)
            bad_row = int(torch.nonzero(c.ids == 1)[0])
            c.x[bad_row, 3] = nan
            c.dy[bad_row, 5] = inf
            c.down[2, 1, 7] = inf
            c.up[2, 0, 9] = nan
            hidden = torch.empty(M, 12, device="cuda")
            out = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base, hidden=hidden)
            fine = (c.ids != 2)
            fine[bad_row] = False
            assert torch.equal(out[fine], clean[fine]) and not out[bad_row].isfinite().any() and bool(out[c.ids == 2][:, 9].isnan().all())
            dx, d_down, d_up = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales)
            assert torch.equal(dx[fine], want[0][fine])
            for a in (0, 3):
                assert torch.equal(d_down[a], want[1][a]) and torch.equal(d_up[a], want[2][a])
            assert not d_down[1][:, 3].isfinite().any() and not d_up[1][:, 5].isfinite().any()


def test_gradients_against_differences():
    """out is linear in each of x, down and up: a central difference of binary64 sums is the derivative itself."""
    c = Case(50, 40, 48, 6, 3, F32, F32, F32, "requests")
    hidden = torch.empty(50, 6, device="cuda")
    mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, hidden=hidden)
    got = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales)

    def total(x, down, up):
        s = c.scales[c.at].double() * c.real
        t = torch.stack([down[a] @ v for a, v in zip(c.at.tolist(), x)])
        return sum(float(f * (h @ up[a]) @ d) for f, h, a, d in zip(s, t, c.at.tolist(), c.dy.double()))
    args = [c.x.double(), c.down.double(), c.up.double()]
    g = torch.Generator("cuda").manual_seed(4)
    for i, grad in enumerate(got):
        way = torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64)
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + way, args[i] - way
        slope = (total(*plus) - total(*minus)) / 2
        assert abs(slope - float((grad.double() * way).sum())) <= 1e-5 * float((grad.double() * way).abs().sum())


def test_rows_past_32_bits():
    M, K, N, wide = 2100, 48, 56, 1 << 20  # places of rows up to 2.2e9
    c = Case(M, K, N, 5, 2, BF16, BF16, BF16, "requests")
    want = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base)
    x = torch.zeros(M, wide, dtype=BF16, device="cuda")
    x[:, :K] = c.x
    out = torch.zeros(M, wide, dtype=BF16, device="cuda")
    hidden = torch.empty(M, 5, device="cuda")
    mkq.mkq_low_rank_adapters(x[:, :K], c.ids, c.down, c.up, c.scales, base=c.base, out=out[:, :N], hidden=hidden)
    assert torch.equal(out[:, :N], want) and not out[:, N:].any()
    a = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales)
    x2 = torch.zeros(M, wide, dtype=BF16, device="cuda")
    x2[:, :N] = c.dy
    b = mkq.mkq_low_rank_adapters_gradient(x2[:, :N], x[:, :K], c.ids, hidden, c.down, c.up, c.scales, dx=out[:, :K])
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_no_rows():
    x, dy, ids = torch.zeros(0, 40, device="cuda"), torch.zeros(0, 48, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    down, up, hidden = torch.zeros(3, 4, 40, device="cuda"), torch.zeros(3, 4, 48, device="cuda"), torch.zeros(0, 4, device="cuda")
    assert mkq.mkq_low_rank_adapters(x, ids, down, up).shape == (0, 48)
    d_down, d_up = torch.ones(3, 4, 40, device="cuda"), torch.ones(3, 4, 48, device="cuda")
    mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up, d_down=d_down, d_up=d_up, accumulate=True)
    assert bool((d_down == 1).all()) and bool((d_up == 1).all())
    mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up, d_down=d_down, d_up=d_up)
    assert not d_down.any() and not d_up.any()


@pytest.mark.parametrize("M,K,N,rank,R", [(16, 768, 768, 8, 16), (1, 4096, 1024, 16, 4), (700, 520, 264, 12, 3)])
def test_equal_calls_streams_and_graph_replays(M, K, N, rank, R):
    c = Case(M, K, N, rank, R, F16, F16, F16, "mixed")
    ws = torch.empty(mkq.mkq_low_rank_adapters_workspace_bytes(M, K, N, rank, R) + 16, dtype=torch.uint8, device="cuda")
    wg = torch.empty(mkq.mkq_low_rank_adapters_gradient_workspace_bytes(M, K, N, rank, R), dtype=torch.uint8, device="cuda")
    hidden = torch.empty(M, rank, device="cuda")

    def run(stream=None, ws=ws, wg=wg, hidden=hidden):
        out = mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base, hidden=hidden, workspace=ws, stream=stream)
        return [out, hidden, *mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales, workspace=wg, stream=stream)]
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = run()
    side = torch.cuda.Stream()
    for i in range(3):
        d = Case(M, K, N, rank, R, F16, F16, F16, "requests", seed=20 + i)
        for name in ("x", "dy", "ids", "down", "up", "base"):
            getattr(c, name).copy_(getattr(d, name))
        ws.fill_(0x5A)
        wg.fill_(0x5A)
        want = [t.clone() for t in run()]
        ws.fill_(0xFF)
        wg.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)), i
        side.wait_stream(torch.cuda.current_stream())
        other = run(side, None, None, torch.empty_like(hidden))
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other, want)), i


@pytest.mark.parametrize("M", [5, 700])
def test_some_of_the_gradients(M):
    """Each of dx, d_down and d_up without the others, what only these need being absent: the bits of the call that makes all."""
    c = Case(M, 72, 88, 7, 3, BF16, BF16, BF16, "requests")
    hidden = torch.randn(M, 7, device="cuda") * c.real[:, None]
    lib, stream = mkq.load(), torch.cuda.current_stream().cuda_stream
    n = mkq.mkq_low_rank_adapters_gradient_workspace_bytes(M, 72, 88, 7, 3)
    all_dx, all_down, all_up = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales)
    _, one_down, _ = mkq.mkq_low_rank_adapters_gradient(c.dy, c.x, c.ids, hidden, c.down, c.up, c.scales, want_dx=False)
    for name, want in (("dx", all_dx), ("d_down", one_down), ("d_up", all_up)):
        got, ws = torch.full_like(want, 7.0), torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
        at = lambda t, needed: t.data_ptr() if name in needed else None  # noqa: E731
        status = lib.mkq_low_rank_adapters_gradient(
            c.dy.data_ptr(), 2, 88, at(c.x, ("d_down",)), 2, 72, None, 0, c.ids.data_ptr(), at(hidden, ("d_up",)), M, 72, 88, 7, 3,
            at(c.down, ("dx",)), at(c.up, ("dx", "d_down")), 2, c.scales.data_ptr(), None, 0, at(got, ("dx",)), 2, 72,
            at(got, ("d_down",)), at(got, ("d_up",)), 0, 0, ws.data_ptr(), n, stream)
        assert status == mkq.MKQ_OK, name
        assert torch.equal(got, want), name


def test_two_calls_at_once():
    """Two streams, a workspace each, against the same calls one after the other."""
    cases = [Case(900, 520, 264, 12, 3, F16, F16, F16, "requests", seed=s) for s in (1, 2)]
    want = [mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(10):
        for k, (c, s) in enumerate(zip(cases, streams)):
            got[k].append(mkq.mkq_low_rank_adapters(c.x, c.ids, c.down, c.up, c.scales, base=c.base, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for gs, w in zip(got, want) for g in gs)
