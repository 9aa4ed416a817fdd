"""Token lookups, the table's gradient by sorted tokens, and a run of them with the tied head and the clipping, against plain
implementations in 64 bits.

A lookup is a product (from nibbles two) in binary32 and one rounding: torch computes the same bits.  A gradient's row of n tokens
is a binary32 sum of n terms in some order, one scaling (accumulating: one fused multiply-add) and one rounding to its type: off
by at most n 2^-24 sum |dy| |scale|, 2^-24 of the result, and half a step of the type."""
import math

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


def some_tokens(M, V, seed, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    t = (V ** torch.rand(M, generator=g, dtype=torch.float64)).long() - 1
    return torch.randperm(V, generator=g)[t.clamp(0, V - 1)].to(dtype)


@pytest.mark.parametrize("out", list(T))
@pytest.mark.parametrize("tt", list(T))
@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (7, 10, 7), (33, 500, 8), (440, 3000, 312), (300, 1000, 768), (5, 9, 1001), (19, 40, 2056), (3, 5, 2500)])
def test_lookup(mkq, M, V, D, tt, out):
    table = torch.randn(V, D, generator=torch.Generator().manual_seed(D)).to(T[tt])
    for dtype, scale in ((torch.int32, 1.0), (torch.int64, math.sqrt(D))):
        t = some_tokens(M, V, M + V, dtype)
        got = mkq.mkq_embedding(t.cuda(), table.cuda(), scale, code(mkq, out))
        want = (table[t.long()].float() * torch.tensor(scale, dtype=torch.float32)).to(T[out])
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("out", list(T))
@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (7, 10, 7), (33, 500, 32), (200, 900, 312), (300, 1000, 768), (19, 40, 2049)])
def test_lookup_int4(mkq, M, V, D, out, group):
    g = torch.Generator().manual_seed(D)
    width = -(-D // 32) * 32
    codes = torch.randint(-8, 8, (V, width), generator=g)
    Wq = ((codes[:, 0::2] % 16) + 16 * (codes[:, 1::2] % 16)).to(torch.uint8)
    s = torch.rand(V, -(-D // group), generator=g) * 0.01
    t = some_tokens(M, V, M)
    got = mkq.mkq_embedding_int4_group(t.cuda(), Wq.cuda(), s.cuda(), V, D, group, 1.7, code(mkq, out))
    rows = codes[:, :D].float() * s.repeat_interleave(group, 1)[:, :D]
    assert torch.equal(got.cpu(), (rows[t] * torch.tensor(1.7)).to(T[out]))


@pytest.mark.parametrize("four", [False, True])
def test_tokens_outside_the_table_give_zeros(mkq, four):
    V, D = 50, 64
    t = torch.tensor([3, -1, 50, 49, -(2 ** 31), 2 ** 31 - 1, 0], dtype=torch.int32)
    far = torch.tensor([3, 2 ** 32 + 3, -(2 ** 32) + 3, 49, 2 ** 62, -(2 ** 63), 0])
    table = torch.full((V, D), float("inf"))
    table[3] = 2.0
    if four:
        Wq, s = mkq.mkq_pack_weights_int4_group(torch.where(table.isinf(), 1.0, table).cuda(), 32)
        look = lambda t: mkq.mkq_embedding_int4_group(t.cuda(), Wq, s, V, D, 32).cpu()
    else:
        look = lambda t: mkq.mkq_embedding(t.cuda(), table.cuda()).cpu()
    for tokens in (t, far):
        got = look(tokens)
        zero = (got == 0).all(1)
        assert zero.tolist() == [False, True, True, False, True, True, False]
        assert bool((got[0] == got[0, 0]).all())


@pytest.mark.parametrize("ld_t,ld_o", [(24, 32), (21, 32), (24, 27), (19, 23)])
def test_lookup_rows_with_gaps(mkq, ld_t, ld_o):
    M, V, D = 70, 30, 19
    for tt in T:
        wide = torch.full((V, ld_t), float("nan"), dtype=T[tt])
        wide[:, :D] = torch.randn(V, D, generator=torch.Generator().manual_seed(1)).to(T[tt])
        room = torch.full((M + 1, ld_o), -5.0, dtype=T[tt], device="cuda")
        t = some_tokens(M, V, 3, torch.int32)
        got = mkq.mkq_embedding(t.cuda(), wide.cuda()[:, :D], out_dtype=code(mkq, tt), out=room[:M, :D])
        assert torch.equal(got.cpu(), wide[t.long(), :D])
        assert bool((room[:M, D:] == -5).all()) and bool((room[M] == -5).all())


def test_lookup_past_32_bits(mkq):
    """A table of more than 2^31 values, and a table of nibbles of more than 2^31 bytes' worth of values"""
    V, D = 70000, 32768
    table = torch.empty(V, D, dtype=torch.float16, device="cuda")
    rows = torch.tensor([0, 1, 65535, 65536, 69999])
    for r in rows.tolist():
        table[r] = torch.arange(D, device="cuda").remainder(1000).half() + r % 7
    got = mkq.mkq_embedding(rows.cuda(), table)
    assert torch.equal(got, table[rows.cuda()])
    del table, got
    Wq = torch.empty(V, D // 2, dtype=torch.uint8, device="cuda")
    s = torch.ones(V, D // 128, device="cuda")
    for r in rows.tolist():
        Wq[r] = (r % 7) * 17 + 1
    got = mkq.mkq_embedding_int4_group(rows.cuda(), Wq, s, V, D, 128, 1.0, mkq.MKQ_F16).cpu()
    for i, r in enumerate(rows.tolist()):
        pair = torch.tensor([(r % 7) + 1, r % 7])
        assert torch.equal(got[i], torch.where(pair > 7, pair - 16, pair).half().repeat(D // 2))


# ---- gradient --------------------------------------------------------------------------------------------------------------
def check_gradient(got, t, dy, V, scale, padding=-1, start=None):
    keep = (t >= 0) & (t < V) & (t != padding)
    t, dy = t[keep].long(), dy[keep].double()
    y = torch.zeros(V, dy.shape[1], dtype=torch.float64).index_add_(0, t, dy) * scale
    S = torch.zeros_like(y).index_add_(0, t, dy.abs()) * abs(scale)
    n = torch.zeros(V, dtype=torch.float64).index_add_(0, t, torch.ones(len(t), dtype=torch.float64))
    tol = n[:, None] * 2.0 ** -24 * S
    if start is not None:
        y = y + start.double()
    tol = tol + 2.0 ** -24 * (y.abs() + tol)
    info = torch.finfo(got.dtype)
    tol = tol + (y.abs() + tol) * info.eps / 2 + info.smallest_normal * info.eps / 2
    none = n == 0
    if start is None:
        assert bool((got.cpu()[none] == 0).all())
    else:
        assert torch.equal(got.cpu()[none], start[none])
    off = (got.cpu().double() - y).abs()
    assert bool((off <= tol)[~none].all()), float((off / tol)[~none].max())


SIZES = [(1, 1, 1), (1, 100, 33), (9, 4, 8), (100, 60, 312), (513, 200, 40), (1024, 511, 16), (3000, 512, 24), (4096, 30522, 64), (5000, 3, 20),
         (2500, 300000, 8), (700, 1000, 2100)]


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("f16", "f32"), ("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,V,D", SIZES)
def test_gradient(mkq, M, V, D, dt, gt):
    g = torch.Generator().manual_seed(M + D)
    dy = torch.randn(M, D, generator=g).to(T[dt])
    for bits, scale, padding in ((torch.int32, 1.0, -1), (torch.int64, -1.5, 0)):
        t = some_tokens(M, V, M, bits)
        t[torch.rand(M, generator=g) < 0.1] = -100
        t[torch.rand(M, generator=g) < 0.2] = 0
        room = torch.full((V + 1, D), -3.0, dtype=T[gt], device="cuda")
        got = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, scale, code(mkq, gt), padding_token=padding, grad=room[:V])
        check_gradient(got, t, dy, V, scale, padding)
        assert bool((room[V] == -3).all())
        again = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, scale, code(mkq, gt), padding_token=padding)
        assert torch.equal(got, again)
        start = torch.randn(V, D, generator=g).to(T[gt])
        added = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, scale, code(mkq, gt), padding_token=padding, grad=start.cuda(), accumulate=True)
        check_gradient(added, t, dy, V, scale, padding, start)


@pytest.mark.parametrize("tokens", ["same", "two", "none", "all_outside", "ascending", "descending"])
@pytest.mark.parametrize("M", [1, 8, 9, 64, 1000, 9000, 70000])
def test_gradient_of_extreme_batches(mkq, M, tokens):
    V, D = 40000, 16
    t = {"same": torch.full((M,), 777), "two": torch.arange(M) % 2 + 39998, "none": torch.full((M,), 5), "all_outside": torch.full((M,), V),
         "ascending": torch.arange(M) % V, "descending": V - 1 - torch.arange(M) % V}[tokens]
    dy = torch.randn(M, D, generator=torch.Generator().manual_seed(M))
    padding = 5 if tokens == "none" else -1
    got = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, padding_token=padding)
    check_gradient(got, t, dy, V, 1.0, padding)


@pytest.mark.parametrize("M,V,D", [(300000, 1000, 8), (300000, 200000, 4), (65536, 30522, 32), (12288, 5000, 24), (12289, 5000, 24), (1200000, 90, 8)])
def test_gradient_of_long_batches(mkq, M, V, D):
    t = some_tokens(M, V, 1, torch.int32)
    dy = torch.randn(M, D, generator=torch.Generator().manual_seed(2))
    check_gradient(mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V), t, dy, V, 1.0)


def test_gradient_of_whole_numbers_is_exact_and_ordered(mkq):
    M, V, D = 20000, 150, 24
    t = some_tokens(M, V, 5)
    dy = torch.randint(-50, 51, (M, D), generator=torch.Generator().manual_seed(6)).float()
    got = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V)
    assert torch.equal(got.cpu(), torch.zeros(V, D).index_add_(0, t, dy))


@pytest.mark.parametrize("ld_y,ld_g", [(24, 32), (21, 24), (24, 21), (19, 23)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_rows_with_gaps(mkq, ld_y, ld_g, accumulate):
    M, V, D = 400, 30, 19
    for dt in T:
        wide = torch.full((M, ld_y), float("nan"), dtype=T[dt])
        wide[:, :D] = torch.randn(M, D, generator=torch.Generator().manual_seed(1)).to(T[dt])
        room = torch.full((V + 1, ld_g), -5.0, dtype=T[dt], device="cuda")
        t = some_tokens(M, V, 3, torch.int32)
        got = mkq.mkq_embedding_gradient(t.cuda(), wide.cuda()[:, :D], V, 1.0, code(mkq, dt), grad=room[:V, :D], accumulate=accumulate)
        check_gradient(got, t, wide[:, :D], V, 1.0, start=torch.full((V, D), -5.0, dtype=T[dt]) if accumulate else None)
        assert bool((room[:V, D:] == -5).all()) and bool((room[V] == -5).all())


@pytest.mark.parametrize("V,D", [(1, 1), (1, 7), (2, 4), (3, 5), (9, 33), (5000, 39)])
@pytest.mark.parametrize("gt", ["f32", "f16", "bf16"])
def test_gradient_rows_of_any_length_without_gaps(mkq, V, D, gt):
    """Rows that begin at every alignment: all of them are written, nothing beside them; a gradient that is not aligned itself is refused"""
    t = torch.tensor([V - 1, 0, -100, V // 2])
    dy = torch.randn(4, D, generator=torch.Generator().manual_seed(D)).to(T[gt])
    for none in (False, True):
        room = torch.full((V * D + 32,), -5.0, dtype=T[gt], device="cuda")
        grad = room[16:16 + V * D].view(V, D)
        tokens = torch.full((4,), -100) if none else t
        mkq.mkq_embedding_gradient(tokens.cuda(), dy.cuda(), V, 1.0, code(mkq, gt), grad=grad)
        check_gradient(grad, tokens, dy, V, 1.0)
        assert bool((room[:16] == -5).all()) and bool((room[16 + V * D:] == -5).all())
    with pytest.raises(mkq.MkqError, match="aligned"):
        mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, 1.0, code(mkq, gt), grad=room[17:17 + V * D].view(V, D))


@pytest.mark.parametrize("M", [4095, 4096, 4097, 4160, 6000])
def test_gradient_at_both_ways_to_rank(mkq, M):
    V, D = 900, 24
    t = some_tokens(M, V, M)
    t[::7] = 11
    dy = torch.randn(M, D, generator=torch.Generator().manual_seed(3))
    check_gradient(mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, padding_token=0), t, dy, V, 1.0, 0)


def test_gradient_past_32_bits(mkq):
    """A gradient, then gradients' rows, of more than 2^31 values"""
    V, D = 70000, 32768
    t = torch.tensor([0, 69999, 65536, 69999, 1])
    dy = torch.randint(-9, 10, (5, D), generator=torch.Generator().manual_seed(1)).half()
    grad = torch.full((V, D), 3.0, dtype=torch.float16, device="cuda")
    mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, 1.0, mkq.MKQ_F16, grad=grad)
    rows = {0: dy[0], 69999: dy[1] + dy[3], 65536: dy[2], 1: dy[4]}
    for r, want in rows.items():
        assert torch.equal(grad[r].cpu(), want)
    counts = torch.count_nonzero(grad, dim=1).cpu()
    assert all(int(counts[r]) == int(torch.count_nonzero(w)) for r, w in rows.items()) and int(counts.sum()) == sum(int(torch.count_nonzero(w)) for w in rows.values())
    del grad
    M = 70000
    t = torch.arange(M) % 3
    dy = torch.zeros(M, D, dtype=torch.float16, device="cuda")
    dy[::1000, 5] = 2.0
    dy[M - 1] = 1.0
    got = mkq.mkq_embedding_gradient(t.cuda(), dy, 4)
    want = torch.zeros(4, D)
    for i in range(0, M, 1000):
        want[i % 3, 5] += 2.0
    want[(M - 1) % 3] += 1.0
    assert torch.equal(got.cpu(), want)


def test_gradient_of_no_tokens(mkq):
    grad = torch.full((9, 20), 4.0, device="cuda")
    t, dy = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, 20, device="cuda")
    assert bool((mkq.mkq_embedding_gradient(t, dy, 9, grad=grad, accumulate=True) == 4).all())
    assert bool((mkq.mkq_embedding_gradient(t, dy, 9, grad=grad) == 0).all())


def test_gradient_keeps_nan_and_infinity_in_their_rows(mkq):
    M, V, D = 600, 70, 16
    t = some_tokens(M, V, 7)
    t[5] = 69
    dy = torch.randn(M, D, generator=torch.Generator().manual_seed(8))
    clean = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V).cpu()
    dy[5, 3], dy[10, 4] = float("nan"), float("inf")
    got = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V).cpu()
    assert math.isnan(float(got[69, 3])) and math.isinf(float(got[t[10], 4]))
    got[69, 3], got[t[10], 4] = clean[69, 3], clean[t[10], 4]
    assert torch.equal(got, clean)


def test_gradient_against_differences_of_the_lookup(mkq):
    """L = sum dy * lookup(table): linear, so L(table + h) - L(table) = <gradient, h>; whole numbers make both sides exact"""
    M, V, D = 900, 200, 40
    g = torch.Generator().manual_seed(9)
    t = some_tokens(M, V, 4).cuda()
    dy = torch.randint(-9, 10, (M, D), generator=g).float().cuda()
    table = torch.randint(-20, 21, (V, D), generator=g).float().cuda()
    grad = mkq.mkq_embedding_gradient(t, dy, V, 4.0).double()
    loss = lambda tab: (mkq.mkq_embedding(t, tab, 4.0).double() * dy.double()).sum()
    for _ in range(5):
        h = torch.randint(-3, 4, (V, D), generator=g).float().cuda()
        assert float(loss(table + h) - loss(table)) == float((grad * h.double()).sum())


def test_streams_and_graphs(mkq):
    """Two calls at once on two streams with workspaces of their own, then both captured and replayed with new inputs"""
    V, D, M = 3000, 64, 2500
    streams = [torch.cuda.Stream() for _ in range(2)]
    ins = [(some_tokens(M, V, i).cuda(), torch.randn(M, D, generator=torch.Generator().manual_seed(i)).cuda()) for i in range(2)]
    torch.cuda.synchronize()
    outs = [mkq.mkq_embedding_gradient(t, dy, V, stream=s) for (t, dy), s in zip(ins, streams)]
    torch.cuda.synchronize()
    for (t, dy), got in zip(ins, outs):
        check_gradient(got, t.cpu(), dy.cpu(), V, 1.0)
    t, dy = ins[0]
    grad, rows = torch.empty(V, D, device="cuda"), torch.empty(M, D, device="cuda")
    ws = torch.empty(mkq.mkq_embedding_gradient_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")

    def run():
        mkq.mkq_embedding_gradient(t, dy, V, grad=grad, workspace=ws)
        mkq.mkq_embedding(t, grad, 0.5, out=rows)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(2, 5):
        t.copy_(some_tokens(M, V, i))
        dy.copy_(torch.randn(M, D, generator=torch.Generator().manual_seed(i)))
        run()
        torch.cuda.synchronize()
        want = grad.clone(), rows.clone()
        grad.fill_(7)
        rows.fill_(7)
        ws.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want[0]) and torch.equal(rows, want[1])


def test_a_tied_table_from_lookup_to_update(mkq):
    """The table of an encoder, as it is used: packed, looked up from, multiplied with as the head, its gradient accumulated from
    both ends, clipped with the others, applied, packed again."""
    V, D, M, group = 700, 96, 50, 32
    g = torch.Generator().manual_seed(11)
    master = torch.randn(V, D, generator=g).cuda() * 0.05
    bias = torch.randn(V, generator=g).cuda() * 0.1
    t = some_tokens(M, V, 12).cuda()
    Wq, s = mkq.mkq_pack_weights_int4_group(master, group)
    values = mkq.mkq_embedding_int4_group(torch.arange(V, device="cuda"), Wq, s, V, D, group)  # the table that the nibbles stand for
    assert float((values - master).abs().max()) <= float(s.max()) * 0.5 * 1.001  # half a step: abs-max / 7 clips nothing
    h = mkq.mkq_embedding_int4_group(t, Wq, s, V, D, group, math.sqrt(D), mkq.MKQ_F16)
    assert torch.equal(h, (values[t] * torch.tensor(math.sqrt(D), dtype=torch.float32)).half())
    logits = mkq.mkq_linear_int4_group(h, Wq, s, bias, V, D, group, mkq.MKQ_F32)
    exact = h.double().cpu() @ values.double().cpu().T + bias.double().cpu()
    assert float((logits.double().cpu() - exact).abs().max()) <= (D + 10) * 2.0 ** -23 * float((h.double().abs().cpu() @ values.double().abs().cpu().T).max() + 1)
    p = torch.softmax(logits.double(), -1)
    p[torch.arange(M), t] -= 1.0  # the loss' gradient with respect to the logits, tokens as targets
    grad = (p.T @ h.double()).float()  # the head's part of the table's gradient
    dh = (p @ values.double()).float()
    start = grad.cpu().clone()
    mkq.mkq_embedding_gradient(t, dh, V, math.sqrt(D), grad=grad, accumulate=True)
    check_gradient(grad, t.cpu(), dh.cpu(), V, math.sqrt(D), start=start)
    dbias = p.sum(0).float()
    before = [grad.double().clone(), dbias.double().clone()]
    norm = mkq.mkq_clip_gradients([grad, dbias], 1.0)
    true = math.sqrt(sum(float(b.square().sum()) for b in before))
    assert true > 1 and abs(float(norm) - true) <= 2.0 ** -23 * true
    for now, b in zip((grad, dbias), before):
        want = b / (true + 1e-6)
        assert bool(((now.double() - want).abs() <= 3 * 2.0 ** -24 * want.abs()).all())
    master -= 0.1 * grad
    Wq2, s2 = mkq.mkq_pack_weights_int4_group(master, group, s)
    assert not torch.equal(Wq2, Wq) and torch.equal(s2, s)


# ---- long batches, where a thread has four rows, and long runs -------------------------------------------------------------
def four_rows_from(D):
    """Tokens from which a thread has four rows, and rows of a workgroup at a time"""
    rows = 256 // min(256, -(-D // 8))
    return rows * 4 * 2048, rows


def lengths_around(D):
    at, rows = four_rows_from(D)
    return [at - 1, at, at + 1, at + rows, at + 4 * rows - 1]


def batch_with_unknown_tokens(M, V, seed, dtype):
    g = torch.Generator("cuda").manual_seed(seed)
    t = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=dtype)
    t[torch.rand(M, generator=g, device="cuda") < 0.2] = V
    t[torch.rand(M, generator=g, device="cuda") < 0.1] = -7
    t[-1] = V - 1
    return t


@pytest.mark.parametrize("D,gap", [(1024, 0), (1024, 8), (2056, 0), (312, 5), (1001, 0), (1001, 7), (2051, 0)])
def test_lookup_of_long_batches(mkq, D, gap):
    """Bits of torch's, at every remainder of four rows a thread; rows with gaps and what lies behind the last one are left alone"""
    V = 300
    for i, M in enumerate(lengths_around(D)):
        kinds = [("f16", "f16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f16", "f32")][i:] + [("bf16", "bf16")]
        for tt, out in kinds[:2]:
            table = torch.randn(V, D, generator=torch.Generator("cuda").manual_seed(D), device="cuda").to(T[tt])
            for dtype, scale in ((torch.int32, 1.0), (torch.int64, 1.7)):
                t = batch_with_unknown_tokens(M, V, M, dtype)
                known = ((t >= 0) & (t < V))[:, None]
                want = torch.where(known, table[t.long().clamp(0, V - 1)].float() * torch.tensor(scale, device="cuda"), 0.0).to(T[out])
                room = torch.full((M + 3, D + gap), -5.0, dtype=T[out], device="cuda")
                got = mkq.mkq_embedding(t, table, scale, code(mkq, out), out=room[:M, :D])
                assert torch.equal(got, want), (M, tt, out)
                assert bool((room[:M, D:] == -5).all()) and bool((room[M:] == -5).all())


@pytest.mark.parametrize("D,gap,group", [(1024, 0, 64), (1024, 8, 128), (2056, 0, 32), (312, 5, 32), (1001, 0, 64), (2051, 0, 128)])
def test_lookup_int4_of_long_batches(mkq, D, gap, group):
    V = 300
    g = torch.Generator("cuda").manual_seed(D)
    codes = torch.randint(-8, 8, (V, -(-D // 32) * 32), generator=g, device="cuda")
    Wq = ((codes[:, 0::2] % 16) + 16 * (codes[:, 1::2] % 16)).to(torch.uint8)
    s = torch.rand(V, -(-D // group), generator=g, device="cuda") * 0.01
    rows = codes[:, :D].float() * s.repeat_interleave(group, 1)[:, :D]
    for i, M in enumerate(lengths_around(D)):
        out, dtype = ["f16", "f32", "bf16"][i % 3], [torch.int32, torch.int64][i % 2]
        t = batch_with_unknown_tokens(M, V, M, dtype)
        known = ((t >= 0) & (t < V))[:, None]
        want = torch.where(known, rows[t.long().clamp(0, V - 1)] * torch.tensor(1.7, device="cuda"), 0.0).to(T[out])
        room = torch.full((M + 3, D + gap), -5.0, dtype=T[out], device="cuda")
        got = mkq.mkq_embedding_int4_group(t, Wq, s, V, D, group, 1.7, code(mkq, out), out=room[:M, :D])
        assert torch.equal(got, want), (M, out)
        assert bool((room[:M, D:] == -5).all()) and bool((room[M:] == -5).all())


def check_exact_gradient(mkq, t, V, D, dt, gt, seed):
    """Whole numbers whose sums stay below 2^24: every order of the additions gives them exactly, so a position that is lost or counted
    twice shows, however long its run is"""
    g = torch.Generator("cuda").manual_seed(seed)
    dy = torch.randint(-9, 10, (len(t), D), generator=g, device="cuda").to(T[dt])
    known = (t >= 0) & (t < V)
    at = "cpu" if V <= 2 ** 20 else "cuda"  # (long runs take seconds there, tables of 2^27 rows here)
    want = torch.zeros(V, D, dtype=torch.float64, device=at).index_add_(0, t[known].long().to(at), dy[known].double().to(at)).cuda()
    assert not bool(known.any()) or int(torch.bincount(t[known].long()).max()) * 9 < 2 ** 24
    assert torch.equal(mkq.mkq_embedding_gradient(t, dy, V, 1.0, code(mkq, gt)), want.to(T[gt]))
    start = torch.randint(-9, 10, (V, D), generator=g, device="cuda").to(T[gt])
    want = want + start.double()
    assert torch.equal(mkq.mkq_embedding_gradient(t, dy, V, 1.0, code(mkq, gt), grad=start, accumulate=True), want.to(T[gt]))


@pytest.mark.parametrize("tokens", ["same", "two", "blocks", "long_and_short", "all_outside", "ascending"])
@pytest.mark.parametrize("M", [1, 8, 9, 63, 65, 1000, 4097, 9000, 12289, 70000, 70001])
@pytest.mark.parametrize("D", [16, 5])
def test_exact_gradient_of_extreme_batches(mkq, M, D, tokens):
    V = 40000
    i = torch.arange(M, device="cuda")
    t = {"same": torch.full_like(i, 777), "two": i % 2 + 39998, "blocks": i // 997, "long_and_short": torch.where(i % 3 == 0, i // 3 % V, 5),
         "all_outside": torch.full_like(i, V), "ascending": i % V}[tokens]
    check_exact_gradient(mkq, t, V, D, "f32", "f32", M)


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("M,V,D", [(300000, 1000, 8), (300000, 200000, 4), (65536, 30522, 32), (12288, 5000, 24), (12289, 5000, 7), (1200000, 90, 8),
                                   (1200000, 90, 3), (20000, 2 ** 18, 8), (100000, 2 ** 18 - 1, 8), (13000, 2 ** 27, 1)])
def test_exact_gradient_of_long_batches(mkq, M, V, D, dt, gt):
    """One digit to four, and runs of up to 180000 positions"""
    t = some_tokens(M, V, 1, torch.int32) if V <= 2 ** 20 else torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(1)).repeat_interleave(3)[:M]
    check_exact_gradient(mkq, t.cuda(), V, D, dt, gt, M + D)


@pytest.mark.parametrize("chunks", [2, 3, 15, 16, 17, 18, 31, 32, 33, 48, 64, 272, 273, 300])
@pytest.mark.parametrize("begin", [0, 1, 8 * 15, 8 * 16 - 1, 8 * 17])
def test_exact_gradient_of_runs_over_any_number_of_chunks(mkq, chunks, begin):
    """A run of one token in a sorted batch that begins and ends at, before and behind the borders of chunks and of their sixteens"""
    for end in (-1, 0, 1):
        n = 8 * chunks + end
        t = torch.cat([torch.arange(begin), torch.full((n,), 5000), 5001 + torch.arange(40)]).int()
        check_exact_gradient(mkq, t.cuda(), 6000, 8, "f32", "f32", chunks)


@pytest.mark.parametrize("dt,gt", [("f32", "f16"), ("f32", "bf16"), ("f16", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("M,V,D", [(700, 100, 24), (700, 100, 21), (13000, 500, 16)])
def test_gradient_between_types(mkq, M, V, D, dt, gt):
    g = torch.Generator().manual_seed(M + D)
    t, dy = some_tokens(M, V, M), torch.randn(M, D, generator=g).to(T[dt])
    check_gradient(mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, -1.5, code(mkq, gt)), t, dy, V, -1.5)
    start = torch.randn(V, D, generator=g).to(T[gt])
    got = mkq.mkq_embedding_gradient(t.cuda(), dy.cuda(), V, -1.5, code(mkq, gt), grad=start.cuda(), accumulate=True)
    check_gradient(got, t, dy, V, -1.5, start=start)


@pytest.mark.parametrize("M,D", [(300, 5000), (300, 5001), (2000, 20000), (2000, 20003)])
def test_exact_gradient_of_long_rows(mkq, M, D):
    """Columns in several rounds of a workgroup, and long runs whose shares of the columns are more than one round"""
    check_exact_gradient(mkq, torch.where(torch.arange(M) % 5 == 0, torch.arange(M) % 7, 2).cuda(), 9, D, "f32", "f32", M + D)


def test_lookups_and_gradient_on_other_streams_at_once(mkq):
    """All three on streams of their own at the same time, inputs made on the current one"""
    M, V, D = 6000, 2000, 320
    table = torch.randn(V, D, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    Wq, s = mkq.mkq_pack_weights_int4_group(table, 32)
    t = torch.randint(0, V, (M,), generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    dy = torch.randint(-9, 10, (M, D), generator=torch.Generator("cuda").manual_seed(3), device="cuda").float()
    calls = [lambda **kw: mkq.mkq_embedding(t, table, 0.3, **kw), lambda **kw: mkq.mkq_embedding_int4_group(t, Wq, s, V, D, 32, 0.3, **kw),
             lambda **kw: mkq.mkq_embedding_gradient(t, dy, V, **kw)]
    want = [f() for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        got = [f(stream=st) for f, st in zip(calls, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
