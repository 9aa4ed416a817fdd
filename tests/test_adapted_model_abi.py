"""Refusals of the log probabilities of tokens, of activations kept in 8 bits, and of the low-rank adapters: status codes of the C ABI before
anything is enqueued, and what the Python binding refuses (no GPU)."""
import ctypes as C
import os

import pytest
import torch

import paper_2203_13483_amd as mkq

P = C.c_void_p(0x1000)      # 16-byte aligned, never dereferenced: validation fails first
Q = C.c_void_p(0x10000000)
ODD = C.c_void_p(0x1004)
VERY_ODD = C.c_void_p(0x1002)
F32, F16, BF16 = mkq.MKQ_F32, mkq.MKQ_F16, mkq.MKQ_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mkq.LIB_PATH):
        from paper_2203_13483_amd import build
        build.build()
    return mkq.load()


def test_log_prob_refusals(lib):
    def call(x=P, dt=F16, ld=100, M=4, V=100, scale=1.0, t=P, bits=64, norm=P, lp=P, H=P, top=5, tt=P, tl=P, ws=None, n=0):
        return lib.mkq_token_log_probs(x, dt, ld, M, V, scale, t, bits, norm, lp, H, top, tt, tl, ws, n, None)
    assert call(dt=mkq.MKQ_I4) == call(dt=9) == call(bits=16) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(V=0), dict(ld=99), dict(top=-1), dict(top=101), dict(V=3, top=4)):
        assert call(**bad) == mkq.MKQ_ERR_SHAPE, bad
    for bad in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** -101, 2.0 ** 101):
        assert call(scale=bad) == mkq.MKQ_ERR_SCALE, bad
    assert call(top=65) == call(V=2 ** 31, ld=2 ** 31) == call(M=2 ** 31) == mkq.MKQ_ERR_UNSUPPORTED
    assert call(x=None) == call(t=None) == call(norm=None) == call(lp=None) == call(H=None) == call(tt=None) == call(tl=None) == mkq.MKQ_ERR_NULL
    assert call(x=ODD) == call(t=ODD) == call(t=VERY_ODD, bits=32) == call(norm=ODD) == call(lp=VERY_ODD) == call(tt=VERY_ODD) == mkq.MKQ_ERR_ALIGN
    assert call(M=0, x=None, t=None) == mkq.MKQ_OK
    big = dict(M=1, V=10 ** 6, ld=10 ** 6)
    need = lib.mkq_token_log_probs_workspace_bytes(1, 10 ** 6, 5)
    assert need > 0 and call(**big) == call(**big, ws=P, n=need - 1) == mkq.MKQ_ERR_WORKSPACE
    assert call(**big, ws=C.c_void_p(0x1008), n=need) == mkq.MKQ_ERR_ALIGN
    assert lib.mkq_token_log_probs_workspace_bytes(5000, 30522, 20) == 0
    assert lib.mkq_token_log_probs_workspace_bytes(-1, 10, 0) == lib.mkq_token_log_probs_workspace_bytes(1, 10, 65) == 0


def test_log_prob_gradient_refusals(lib):
    def call(x=P, dt=F16, ld=100, M=4, V=100, scale=1.0, t=P, bits=64, norm=P, H=None, d=P, h=None, g=Q, gdt=F16, ldg=100):
        return lib.mkq_token_log_probs_gradient(x, dt, ld, M, V, scale, t, bits, norm, H, d, h, g, gdt, ldg, None)
    assert call(dt=mkq.MKQ_I4) == call(gdt=-1) == call(bits=8) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(V=0), dict(ld=99), dict(ldg=99)):
        assert call(**bad) == mkq.MKQ_ERR_SHAPE, bad
    assert call(scale=0.0) == call(scale=float("nan")) == mkq.MKQ_ERR_SCALE
    assert call(x=None) == call(t=None) == call(norm=None) == call(d=None) == call(g=None) == call(h=P) == mkq.MKQ_ERR_NULL
    assert call(x=ODD) == call(g=ODD) == call(norm=ODD) == call(d=VERY_ODD) == call(h=VERY_ODD, H=P) == call(t=ODD) == mkq.MKQ_ERR_ALIGN
    # over the scores, but not exactly: another type, another stride, another place
    assert call(g=P, gdt=F32) == call(g=P, ldg=104) == call(g=C.c_void_p(0x1010)) == mkq.MKQ_ERR_UNSUPPORTED
    assert call(V=2 ** 31, ld=2 ** 31, ldg=2 ** 31) == call(M=2 ** 31) == mkq.MKQ_ERR_UNSUPPORTED
    assert call(M=0, x=None) == mkq.MKQ_OK


def test_checkpoint_refusals(lib):
    def keep(x=P, dt=F16, M=4, K=100, ld=100, group=64, c=P, s=P):
        return lib.mkq_checkpoint_int8(x, dt, M, K, ld, group, c, s, None)

    def back(c=P, s=P, group=64, M=4, K=100, act=0, o=P, dt=F16, ld=100):
        return lib.mkq_checkpoint_restore(c, s, group, M, K, act, o, dt, ld, None)

    def slope(c=P, s=P, group=64, M=4, K=100, dy=P, dt=F16, ld=100, dx=Q, odt=F16, ldo=100):
        return lib.mkq_checkpoint_gelu_gradient(c, s, group, M, K, dy, dt, ld, dx, odt, ldo, None)
    assert keep(dt=mkq.MKQ_I8) == back(dt=mkq.MKQ_I8) == back(act=2) == slope(dt=5) == slope(odt=-1) == mkq.MKQ_ERR_DTYPE
    for f in (keep, back, slope):
        for bad in (dict(M=-1), dict(K=0), dict(ld=99), dict(group=0), dict(group=16), dict(group=256)):
            assert f(**bad) == mkq.MKQ_ERR_SHAPE, (f, bad)
        assert f(M=0) == mkq.MKQ_OK
        assert f(c=None) == f(s=None) == mkq.MKQ_ERR_NULL
        assert f(c=ODD) == f(s=VERY_ODD) == mkq.MKQ_ERR_ALIGN
        assert f(M=2 ** 31) == f(K=2 ** 31, ld=2 ** 31, **({"ldo": 2 ** 31} if f is slope else {})) == mkq.MKQ_ERR_UNSUPPORTED
    assert slope(ldo=99) == mkq.MKQ_ERR_SHAPE
    assert keep(x=None) == back(o=None) == slope(dy=None) == slope(dx=None) == mkq.MKQ_ERR_NULL
    assert keep(x=ODD) == back(o=ODD) == slope(dy=ODD) == slope(dx=ODD) == mkq.MKQ_ERR_ALIGN
    assert slope(dx=P, odt=F32) == slope(dx=P, ldo=104) == slope(dx=C.c_void_p(0x1010)) == mkq.MKQ_ERR_UNSUPPORTED
    assert lib.mkq_checkpoint_bytes(3, 33) == 3 * 64 and lib.mkq_checkpoint_bytes(-1, 3) == lib.mkq_checkpoint_bytes(1, 0) == 0


def test_adapter_refusals(lib):
    def fwd(x=P, dt=F16, ldx=64, a=P, M=4, K=64, N=32, rank=8, R=2, down=P, up=P, w=F16, scales=None, base=None, ldb=32, out=Q, odt=F16, ldo=32,
            hidden=None, ws=P, n=1 << 20):
        return lib.mkq_low_rank_adapters(x, dt, ldx, a, M, K, N, rank, R, down, up, w, scales, base, ldb, out, odt, ldo, hidden, ws, n, None)
    assert fwd(dt=mkq.MKQ_I8) == fwd(w=mkq.MKQ_I4) == fwd(odt=-1) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(K=0), dict(N=0), dict(rank=0), dict(R=0), dict(ldx=63), dict(ldo=31), dict(base=P, ldb=31)):
        assert fwd(**bad) == mkq.MKQ_ERR_SHAPE, bad
    assert fwd(K=7) == fwd(N=7) == fwd(ldo=2 ** 25 + 8) == fwd(base=P, ldb=2 ** 25 + 8) == mkq.MKQ_ERR_UNSUPPORTED
    assert fwd(rank=257) == fwd(R=2 ** 23) == fwd(M=2 ** 31) == fwd(K=2 ** 31, ldx=2 ** 31) == fwd(N=2 ** 31, ldo=2 ** 31) == mkq.MKQ_ERR_UNSUPPORTED
    assert fwd(x=None) == fwd(a=None) == fwd(down=None) == fwd(up=None) == fwd(out=None) == mkq.MKQ_ERR_NULL
    for bad in (dict(x=ODD), dict(a=VERY_ODD), dict(down=ODD), dict(up=ODD), dict(scales=VERY_ODD), dict(base=ODD), dict(out=ODD), dict(hidden=VERY_ODD), dict(ws=ODD, M=100)):
        assert fwd(**bad) == mkq.MKQ_ERR_ALIGN, bad
    assert fwd(base=Q, ldb=40) == fwd(base=C.c_void_p(0x10000010)) == mkq.MKQ_ERR_UNSUPPORTED
    assert lib.mkq_low_rank_adapters_workspace_bytes(4, 64, 32, 8, 2) == 0  # few rows in one launch
    need = lib.mkq_low_rank_adapters_workspace_bytes(100, 64, 32, 8, 2)
    assert need >= 100 * 8 * 4 and fwd(M=100, ws=None) == fwd(M=100, n=need - 1) == mkq.MKQ_ERR_WORKSPACE
    assert fwd(M=0, x=None, ws=None) == mkq.MKQ_OK
    assert lib.mkq_low_rank_adapters_workspace_bytes(4, 64, 32, 300, 2) == lib.mkq_low_rank_adapters_workspace_bytes(-4, 64, 32, 3, 2) == 0

    X, DX = C.c_void_p(0x20000000), C.c_void_p(0x30000000)

    def bwd(dy=Q, dt=F16, ldy=32, x=X, xt=F16, ldx=64, steps=None, group=0, a=P, hidden=P, M=4, K=64, N=32, rank=8, R=2, down=P, up=P, w=F16, scales=None,
            base=None, ldb=64, dx=DX, dxt=F16, ldd=64, dd=P, du=P, g=F32, acc=0, ws=P, n=1 << 20):
        return lib.mkq_low_rank_adapters_gradient(dy, dt, ldy, x, xt, ldx, steps, group, a, hidden, M, K, N, rank, R, down, up, w, scales, base, ldb, dx, dxt,
                                                  ldd, dd, du, g, acc, ws, n, None)
    assert bwd(dt=mkq.MKQ_I8) == bwd(xt=mkq.MKQ_I4) == bwd(w=9) == bwd(dxt=mkq.MKQ_I8) == bwd(g=mkq.MKQ_I8) == mkq.MKQ_ERR_DTYPE
    for bad in (dict(M=-1), dict(rank=0), dict(R=0), dict(ldy=31), dict(ldx=63), dict(ldd=63), dict(base=P, ldb=63), dict(xt=mkq.MKQ_I8, steps=P, group=16)):
        assert bwd(**bad) == mkq.MKQ_ERR_SHAPE, bad
    for bad in (dict(dy=None), dict(x=None), dict(a=None), dict(hidden=None), dict(down=None), dict(up=None), dict(xt=mkq.MKQ_I8, group=32),
                dict(dx=None, dd=None, du=None)):
        assert bwd(**bad) == mkq.MKQ_ERR_NULL, bad
    for bad in (dict(dy=ODD), dict(x=ODD), dict(a=VERY_ODD), dict(hidden=VERY_ODD), dict(dx=ODD), dict(dd=ODD), dict(du=ODD), dict(base=ODD), dict(ws=ODD),
                dict(steps=VERY_ODD, xt=mkq.MKQ_I8, group=32)):
        assert bwd(**bad) == mkq.MKQ_ERR_ALIGN, bad
    # dx over what is read behind it
    assert bwd(dx=Q) == bwd(dx=X) == bwd(base=DX, ldb=72) == bwd(rank=257) == mkq.MKQ_ERR_UNSUPPORTED
    need = lib.mkq_low_rank_adapters_gradient_workspace_bytes(4, 64, 32, 8, 2)
    assert lib.mkq_low_rank_adapters_gradient_workspace_bytes(0, 64, 32, 8, 2) > 0 and bwd(M=0, ws=None) == mkq.MKQ_ERR_WORKSPACE
    assert need > 0 and bwd(ws=None) == bwd(n=need - 1) == mkq.MKQ_ERR_WORKSPACE


def test_binding_refuses_what_it_would_read_wrongly():
    x, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: mkq.mkq_token_log_probs(x.T, t), lambda: mkq.mkq_token_log_probs(x, t[:3]), lambda: mkq.mkq_token_log_probs(x, t, 1.0, 11),
                 lambda: mkq.mkq_token_log_probs(x.double(), t), lambda: mkq.mkq_token_log_probs(x, t.float()), lambda: mkq.mkq_token_log_probs(x, t),
                 lambda: mkq.mkq_checkpoint_int8(x, 16), lambda: mkq.mkq_checkpoint_int8(x[:, ::2], 32), lambda: mkq.mkq_checkpoint_int8(x, 32),
                 lambda: mkq.mkq_checkpoint_restore(torch.zeros(4, 10, dtype=torch.int8), torch.ones(4, 1), 10, 32),
                 lambda: mkq.mkq_checkpoint_restore(torch.zeros(4, 32, dtype=torch.int8), torch.ones(4, 2), 10, 32),
                 lambda: mkq.mkq_checkpoint_restore(torch.zeros(4, 32, dtype=torch.int8), torch.ones(4, 1), 10, 32),
                 lambda: mkq.mkq_checkpoint_gelu_gradient(torch.zeros(3, 32, dtype=torch.int8), torch.ones(3, 1), x, 32)):
        with pytest.raises(ValueError):
            call()
    r = mkq.TokenLogProbs()
    r.normalizers, r.entropies = torch.zeros(4, 2), torch.zeros(4)
    for kw in (dict(d=torch.zeros(3)), dict(d=torch.zeros(4, dtype=torch.float16)), dict(d=torch.zeros(4), grad_dtype=mkq.MKQ_I8),
               dict(d=torch.zeros(4), d_entropies=torch.zeros(5)), dict(d=torch.zeros(4))):
        with pytest.raises(ValueError):
            mkq.mkq_token_log_probs_gradient(x, t, r, kw.pop("d"), **kw)
    ids, down, up = torch.zeros(4, dtype=torch.int32), torch.zeros(2, 3, 10), torch.zeros(2, 3, 12)
    dy, hidden = torch.zeros(4, 12), torch.zeros(4, 3)
    for call in (lambda: mkq.mkq_low_rank_adapters(x, ids.long(), down, up), lambda: mkq.mkq_low_rank_adapters(x, ids[:3], down, up),
                 lambda: mkq.mkq_low_rank_adapters(x, ids, down, up.half()), lambda: mkq.mkq_low_rank_adapters(x, ids, down, up[:1]),
                 lambda: mkq.mkq_low_rank_adapters(x, ids, down[:, :, :9], up), lambda: mkq.mkq_low_rank_adapters(x, ids, down, up, torch.ones(3)),
                 lambda: mkq.mkq_low_rank_adapters(x, ids, down, up),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden[:3], down, up),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x[:3], ids, hidden, down, up),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up, accumulate=True),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up, want_dx=False, dx=x),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up, steps=torch.ones(4, 1), group=32),
                 lambda: mkq.mkq_low_rank_adapters_gradient(dy, x, ids, hidden, down, up)):
        with pytest.raises(ValueError):
            call()
