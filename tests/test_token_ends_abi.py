"""Refusals of the group-scaled 4-bit linear, the token lookups, the table's gradient and the gradient clipping: status codes
of the C ABI before anything is enqueued, and what the Python binding refuses (no GPU)."""
import ctypes as C
import os

import pytest
import torch

import paper_2203_13483_amd as mkq

P = C.c_void_p(0x1000)      # 16-byte aligned, never dereferenced: validation fails first
ODD = C.c_void_p(0x1004)
VERY_ODD = C.c_void_p(0x1002)
F32, F16, BF16 = mkq.MKQ_F32, mkq.MKQ_F16, mkq.MKQ_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mkq.LIB_PATH):
        from paper_2203_13483_amd import build
        build.build()
    return mkq.load()


def test_group_pack_refusals(lib):
    def pack(W=P, dt=F32, N=8, K=64, ldw=64, group=32, s_in=None, s_out=P, q=P):
        return lib.mkq_pack_weights_int4_group(W, dt, N, K, ldw, group, s_in, s_out, q, None)
    assert pack(W=None) == pack(s_out=None) == pack(q=None) == mkq.MKQ_ERR_NULL
    assert pack(dt=mkq.MKQ_I4) == pack(dt=-1) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(N=-1), dict(K=0), dict(ldw=63), dict(group=0), dict(group=16), dict(group=256), dict(group=-32)):
        assert pack(**bad) == mkq.MKQ_ERR_SHAPE, bad
    assert pack(W=ODD) == pack(q=ODD) == pack(s_out=VERY_ODD) == pack(s_in=VERY_ODD) == mkq.MKQ_ERR_ALIGN
    assert pack(K=2 ** 31, ldw=2 ** 31) == pack(N=2 ** 31) == pack(N=2 ** 30) == mkq.MKQ_ERR_UNSUPPORTED
    assert pack(N=0, W=None) == mkq.MKQ_OK
    assert lib.mkq_group_weight_bytes(10, 33) == 10 * 32 and lib.mkq_group_weight_bytes(10, 0) == 0
    assert lib.mkq_group_weight_bytes(-1, 32) == 0


def test_group_linear_refusals(lib):
    def lin(x=P, dt=F16, ldx=64, Wq=P, s_w=P, group=32, bias=None, M=4, N=16, K=64, out=P, odt=F32, epi=None):
        return lib.mkq_linear_int4_group(x, dt, ldx, Wq, s_w, group, bias, M, N, K, out, odt, C.byref(epi) if epi else None, None)
    assert lin(x=None) == lin(Wq=None) == lin(s_w=None) == lin(out=None) == mkq.MKQ_ERR_NULL
    assert lin(dt=mkq.MKQ_I8) == lin(odt=mkq.MKQ_I4) == lin(odt=7) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(ldx=63), dict(group=48), dict(group=0)):
        assert lin(**bad) == mkq.MKQ_ERR_SHAPE, bad
    assert lin(x=ODD) == lin(Wq=ODD) == lin(out=ODD) == lin(s_w=VERY_ODD) == lin(bias=VERY_ODD) == mkq.MKQ_ERR_ALIGN
    assert lin(K=2 ** 31, ldx=2 ** 31) == lin(N=2 ** 31) == lin(M=2 ** 31) == lin(M=2 ** 30, N=2 ** 30) == mkq.MKQ_ERR_UNSUPPORTED
    assert lin(M=0, x=None, out=None) == mkq.MKQ_OK
    assert lin(epi=mkq.Epilogue(act=9)) == mkq.MKQ_ERR_DTYPE
    assert lin(epi=mkq.Epilogue(residual=0x1000, residual_dtype=mkq.MKQ_I4)) == mkq.MKQ_ERR_DTYPE
    assert lin(epi=mkq.Epilogue(residual=0x1004)) == mkq.MKQ_ERR_ALIGN
    for kw in (dict(q_out=0x1000), dict(acc_out=0x1000), dict(q_pitch=64)):
        assert lin(epi=mkq.Epilogue(**kw)) == mkq.MKQ_ERR_UNSUPPORTED


def test_lookup_refusals(lib):
    def look(t=P, bits=32, M=4, table=P, dt=F16, V=100, D=64, ldt=64, scale=1.0, out=P, odt=F16, ldo=64):
        return lib.mkq_embedding(t, bits, M, table, dt, V, D, ldt, scale, out, odt, ldo, None)

    def look4(t=P, bits=32, M=4, Wq=P, s_w=P, group=32, V=100, D=64, scale=1.0, out=P, odt=F16, ldo=64):
        return lib.mkq_embedding_int4_group(t, bits, M, Wq, s_w, group, V, D, scale, out, odt, ldo, None)
    for f in (look, look4):
        assert f(t=None) == f(out=None) == mkq.MKQ_ERR_NULL
        assert f(bits=16) == f(odt=mkq.MKQ_I8) == mkq.MKQ_ERR_DTYPE
        for bad in (dict(M=-1), dict(V=0), dict(D=0), dict(ldo=63)):
            assert f(**bad) == mkq.MKQ_ERR_SHAPE, bad
        assert f(out=ODD) == f(t=VERY_ODD) == f(t=ODD, bits=64) == mkq.MKQ_ERR_ALIGN
        assert f(scale=float("nan")) == f(scale=float("inf")) == mkq.MKQ_ERR_SCALE
        assert f(V=2 ** 31) == mkq.MKQ_ERR_UNSUPPORTED
        wide = dict(D=2 ** 31 - 1000, ldo=2 ** 31)
        assert f(**(wide if f is look4 else dict(wide, ldt=2 ** 31))) == mkq.MKQ_ERR_UNSUPPORTED
        assert f(M=0, t=None, out=None) == mkq.MKQ_OK
    assert look(table=None) == look4(Wq=None) == look4(s_w=None) == mkq.MKQ_ERR_NULL
    assert look(dt=mkq.MKQ_I4) == mkq.MKQ_ERR_DTYPE and look(ldt=63) == mkq.MKQ_ERR_SHAPE and look4(group=8) == mkq.MKQ_ERR_SHAPE
    assert look(table=ODD) == look4(Wq=ODD) == look4(s_w=VERY_ODD) == mkq.MKQ_ERR_ALIGN


def test_table_gradient_refusals(lib):
    need = lib.mkq_embedding_gradient_workspace_bytes(4, 64)
    assert need > 0 and lib.mkq_embedding_gradient_workspace_bytes(0, 64) == 0 and lib.mkq_embedding_gradient_workspace_bytes(4, -1) == 0

    def grad(t=P, bits=32, M=4, dy=P, dt=F16, ldy=64, V=100, D=64, scale=1.0, pad=-1, acc=0, g=P, gdt=F32, ldg=64, ws=P, nb=need):
        return lib.mkq_embedding_gradient(t, bits, M, dy, dt, ldy, V, D, scale, pad, acc, g, gdt, ldg, ws, nb, None)
    assert grad(t=None) == grad(dy=None) == grad(g=None) == mkq.MKQ_ERR_NULL
    assert grad(bits=8) == grad(dt=mkq.MKQ_I4) == grad(gdt=5) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(V=0), dict(D=0), dict(ldy=63), dict(ldg=63)):
        assert grad(**bad) == mkq.MKQ_ERR_SHAPE, bad
    assert grad(dy=ODD) == grad(g=ODD) == grad(t=VERY_ODD) == grad(t=ODD, bits=64) == grad(ws=ODD) == mkq.MKQ_ERR_ALIGN
    assert grad(scale=float("nan")) == mkq.MKQ_ERR_SCALE
    assert grad(ws=None) == grad(nb=need - 1) == mkq.MKQ_ERR_WORKSPACE
    assert grad(V=2 ** 31) == grad(M=2 ** 31) == grad(D=2 ** 31 - 1000, ldy=2 ** 31, ldg=2 ** 31) == mkq.MKQ_ERR_UNSUPPORTED
    assert lib.mkq_embedding_gradient_workspace_bytes(4, 2 ** 31 - 1000) == 0


def test_clip_refusals(lib):
    need = lib.mkq_gradient_norm_workspace_bytes(1)
    assert need > 0 and lib.mkq_gradient_norm_workspace_bytes(-1) == 0

    def clip(n=1, at=0x1000, out=0x1000, count=8, dt=F32, mx=1.0, norm=P, ws=P, nb=need, lists=True):
        a, o = (C.c_void_p * 1)(at), (C.c_void_p * 1)(out)
        c, d = (C.c_int64 * 1)(count), (C.c_int32 * 1)(dt)
        if not lists:
            a = o = c = d = None
        r = lib.mkq_clip_gradients(n, a, o, c, d, mx, norm, ws, nb, None)
        if out == at and mx == 1.0:  # the norm alone refuses the same
            assert lib.mkq_gradient_norm(n, a, c, d, norm, ws, nb, None) == r
        return r
    assert clip(norm=None) == clip(lists=False) == clip(at=0, out=0) == clip(out=0) == mkq.MKQ_ERR_NULL
    assert clip(n=-1) == clip(count=-1) == mkq.MKQ_ERR_SHAPE
    assert clip(dt=mkq.MKQ_I4) == mkq.MKQ_ERR_DTYPE
    assert clip(at=0x1002, out=0x1002) == clip(at=0x1001, out=0x1001, dt=F16) == clip(norm=VERY_ODD) == clip(ws=ODD) == mkq.MKQ_ERR_ALIGN
    assert clip(out=0x1002) == mkq.MKQ_ERR_ALIGN
    for bad in (0.0, -1.0, float("nan")):
        assert clip(mx=bad) == mkq.MKQ_ERR_SCALE
    assert clip(ws=None) == clip(nb=need - 1) == mkq.MKQ_ERR_WORKSPACE
    assert clip(count=2 ** 62) == mkq.MKQ_ERR_UNSUPPORTED


def test_binding_refuses_what_it_would_read_wrongly(lib):
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    Wq, s_w = torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(16, 2)
    for call in (lambda: mkq.mkq_linear_int4_group(x, Wq, s_w, None, 16, 64, 32),      # not on a GPU
                 lambda: mkq.mkq_linear_int4_group(x.T, Wq, s_w, None, 16, 4, 32),     # rows that are not contiguous
                 lambda: mkq.mkq_linear_int4_group(x, Wq, s_w, None, 16, 32, 32),      # another K
                 lambda: mkq.mkq_embedding(t, x),
                 lambda: mkq.mkq_embedding(t.float(), x),
                 lambda: mkq.mkq_embedding(torch.zeros(8, dtype=torch.int32)[::2], x),
                 lambda: mkq.mkq_embedding_int4_group(t, Wq, s_w, 16, 64, 32),
                 lambda: mkq.mkq_embedding_gradient(t, x, 100),
                 lambda: mkq.mkq_embedding_gradient(t[:3], x, 100),
                 lambda: mkq.mkq_gradient_norm([]),
                 lambda: mkq.mkq_gradient_norm([x.T]),
                 lambda: mkq.mkq_clip_gradients([x], 1.0),
                 lambda: mkq.mkq_pack_weights_int4_group(x)):
        with pytest.raises(ValueError):
            call()


def test_binding_names_types_that_it_does_not_take(lib):
    """Types that are neither binary32, binary16 nor bfloat16 (the binary64 sums of mkq_scale_gradients among them) are refused by name"""
    x, t, d = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 64, dtype=torch.float64)
    Wq, s_w = torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(16, 2)
    for call in (lambda: mkq.mkq_linear_int4_group(d, Wq, s_w, None, 16, 64, 32),
                 lambda: mkq.mkq_linear_int4_group(x, Wq, s_w, None, 16, 64, 32, mkq.MKQ_I4),
                 lambda: mkq.mkq_linear_int4_group(x, Wq, s_w, None, 16, 64, 32, residual=torch.zeros(4, 16, dtype=torch.float64)),
                 lambda: mkq.mkq_embedding(t, d),
                 lambda: mkq.mkq_embedding(t, x.to(torch.int8)),
                 lambda: mkq.mkq_embedding(t, x, 1.0, 9),
                 lambda: mkq.mkq_embedding_int4_group(t, Wq, s_w, 16, 64, 32, 1.0, mkq.MKQ_I8),
                 lambda: mkq.mkq_embedding_gradient(t, d, 100),
                 lambda: mkq.mkq_embedding_gradient(t, x, 100, 1.0, mkq.MKQ_I4),
                 lambda: mkq.mkq_gradient_norm([x, d]),
                 lambda: mkq.mkq_clip_gradients([x, d], 1.0),
                 lambda: mkq.mkq_pack_weights_int4_group(d)):
        with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
            call()


def test_clip_refuses_results_over_other_tensors(lib):
    """A result written where another tensor is read or written: whole tensors in another order, one twice, parts, between many and
    between types.  (Every call here is refused: the addresses are nobody's.)"""
    def clip(ats, outs, counts, dtypes=None):
        n = len(ats)
        a, o = (C.c_void_p * n)(*ats), (C.c_void_p * n)(*outs)
        c, d = (C.c_int64 * n)(*counts), (C.c_int32 * n)(*(dtypes or [F32] * n))
        return lib.mkq_clip_gradients(n, a, o, c, d, 1.0, P, P, lib.mkq_gradient_norm_workspace_bytes(n), None)
    A, B, D = 0x100000, 0x200000, 0x300000
    for call in (lambda: clip([A, B], [B, A], [8, 8]),                                   # permuted
                 lambda: clip([A, B], [D, A], [8, 8]),
                 lambda: clip([A, A], [A, A], [8, 8]),                                   # twice, in place and not
                 lambda: clip([A, B], [D, D], [8, 8]),
                 lambda: clip([A, A], [A, B], [8, 8]),                                   # in place where another reads
                 lambda: clip([A], [A + 16], [8]),                                       # over a part of itself
                 lambda: clip([A, B], [D, D + 28], [8, 8]),                              # the last value of a result
                 lambda: clip([A, A + 28], [A, A + 28], [8, 8]),
                 lambda: clip([A, D], [A, B], [0x100001 // 4 + 1, 8]),
                 lambda: clip([A, B], [D, D + 8], [8, 8], [F16, F32]),
                 lambda: clip([A + 64 * i for i in range(700)], [A + 64 * (i ^ (i > 600)) for i in range(700)], [16] * 700),
                 lambda: clip([A, 0, B], [B, 0, A], [8, 0, 8])):
        assert call() == mkq.MKQ_ERR_UNSUPPORTED


def test_binding_refuses_workspaces_with_gaps(lib):
    """A view that counts more bytes than lie behind its address, or others' bytes between its own"""
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 21, dtype=torch.uint8)[::2]):
        for call in (lambda: mkq.mkq_embedding_gradient(t, x, 100, workspace=ws),
                     lambda: mkq.mkq_gradient_norm([x], workspace=ws),
                     lambda: mkq.mkq_clip_gradients([x], 1.0, workspace=ws)):
            with pytest.raises(ValueError, match="workspace"):
                call()
