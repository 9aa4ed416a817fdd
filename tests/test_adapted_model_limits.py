"""Limits of the operators of adapted models that the host checks (no GPU): status codes of the C ABI before anything is enqueued."""
import ctypes as C
import os

import pytest

import paper_2203_13483_amd as mkq

P, Q, X = C.c_void_p(0x1000), C.c_void_p(0x10000000), 0x20000000  # 16-byte aligned, never dereferenced: validation fails first
F32, F16 = mkq.MKQ_F32, mkq.MKQ_F16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mkq.LIB_PATH):
        from paper_2203_13483_amd import build
        build.build()
    return mkq.load()


def _adapters(lib, x=X, ldx=768, out=0x30000000, ldo=768, base=None, hidden=None, M=16, K=768, N=768, rank=8, xt=F16, ot=F16, ws=None, n=0):
    """Without room to work in: what is not refused before is a missing workspace, but for few rows, which would run."""
    v = C.c_void_p
    return lib.mkq_low_rank_adapters(v(x), xt, ldx, P, M, K, N, rank, 4, Q, Q, F16, None, v(base) if base else None, ldo, v(out), ot, ldo,
                                     v(hidden) if hidden else None, ws, n, None)


@pytest.mark.parametrize("M", [1, 16, 64, 65, 4096])
def test_results_over_the_rows_they_are_computed_from(lib, M):
    """Workgroups of other columns may still read x where results are written."""
    last = 2 * 768 * M
    for base in (None, X):
        assert _adapters(lib, out=X, base=base, M=M) == mkq.MKQ_ERR_UNSUPPORTED
    for out in (X + 16, X + last - 16, X - last + 16):
        assert _adapters(lib, out=out, M=M) == mkq.MKQ_ERR_UNSUPPORTED, hex(out - X)
    assert _adapters(lib, out=X, ot=F32, M=M) == _adapters(lib, out=X - 4 * 768 * M + 16, ot=F32, M=M) == mkq.MKQ_ERR_UNSUPPORTED
    # hidden values are results, too
    assert _adapters(lib, hidden=X, M=M) == _adapters(lib, hidden=X + last - 4, M=M) == mkq.MKQ_ERR_UNSUPPORTED
    assert _adapters(lib, hidden=0x30000000, M=M) == _adapters(lib, hidden=0x30000000 - 32 * M + 4, M=M) == mkq.MKQ_ERR_UNSUPPORTED
    # columns of one wide matrix that overlap by a vector, where rows follow each other
    if M > 1:
        assert _adapters(lib, ldx=1600, out=X + 2 * 760, ldo=1600, M=M) == _adapters(lib, ldx=1600, out=X + 2 * 840, ldo=1600, M=M) == mkq.MKQ_ERR_UNSUPPORTED


def test_results_beside_the_rows_they_are_computed_from(lib):
    M, last = 4096, 2 * 768 * 4096
    for out in (X + last, X - last):
        assert _adapters(lib, out=out, M=M) == mkq.MKQ_ERR_WORKSPACE
    # columns of one wide matrix, side by side: none is written that is read
    for at in (768, 800, 832):
        assert _adapters(lib, ldx=1600, out=X + 2 * at, ldo=1600, M=M) == _adapters(lib, ldx=1600, out=X - 2 * at, ldo=1600, M=M) == mkq.MKQ_ERR_WORKSPACE
    assert _adapters(lib, ldx=1600, out=X + 2 * 1600 + 2 * 800, ldo=1600, M=M) == mkq.MKQ_ERR_WORKSPACE
    assert _adapters(lib, hidden=X + last, M=M) == _adapters(lib, hidden=X - 32 * M, M=M) == mkq.MKQ_ERR_WORKSPACE


def test_activations_kept_over_what_they_are_made_of(lib):
    """Rows are kept and read back by workgroups side by side: codes, steps and results lie apart."""
    v, M, K, g = C.c_void_p, 100, 256, 64
    x, codes, steps, out = X, X + 0x1000000, X + 0x2000000, X + 0x3000000
    rows, kept, step = 2 * M * K, M * K, 4 * M * (K // g)

    def keep(x=x, c=codes, s=steps, dt=F16):
        return lib.mkq_checkpoint_int8(v(x), dt, M, K, K, g, v(c), v(s), None)

    def back(c=codes, s=steps, o=out, dt=F16):
        return lib.mkq_checkpoint_restore(v(c), v(s), g, M, K, mkq.MKQ_ACT_GELU, v(o), dt, K, None)

    def slope(c=codes, s=steps, o=out, dy=x, dt=F16):
        return lib.mkq_checkpoint_gelu_gradient(v(c), v(s), g, M, K, v(dy), dt, K, v(o), dt, K, None)
    for at in (x, x + 16, x + rows - 16, x - kept + 16):
        assert keep(c=at) == mkq.MKQ_ERR_UNSUPPORTED, hex(at)
    for at in (x, x + rows - 4, x - step + 4, codes, codes + kept - 4, codes - step + 4):
        assert keep(s=at) == mkq.MKQ_ERR_UNSUPPORTED, hex(at)
    for f in (back, slope):
        for at in (codes, codes + kept - 16, codes - rows + 16, steps, steps + step - 16, steps - rows + 16):
            assert f(o=at) == mkq.MKQ_ERR_UNSUPPORTED, hex(at)
        assert f(o=codes, dt=F32) == f(o=codes - 2 * rows + 16, dt=F32) == mkq.MKQ_ERR_UNSUPPORTED
    assert slope(dy=codes, o=codes) == mkq.MKQ_ERR_UNSUPPORTED


def test_adapters_times_rows(lib):
    """Every adapter's rows are found by reading all rows' adapters: so many that a call would hold the GPU for seconds are refused."""
    def call(M, R, dd=0x40000000000, du=0x50000000000, dx=None):
        v = lambda a: C.c_void_p(a) if a else None  # noqa: E731
        return lib.mkq_low_rank_adapters_gradient(v(X), F16, 8, v(0x10000000000), F16, 8, None, 0, P, P, M, 8, 8, 1, R, P, P, F16, None, None, 0, v(dx), F16, 8,
                                                  v(dd), v(du), F32, 0, None, 0, None)
    for M, R in ((2 ** 20, 2 ** 20 + 1), (2 ** 26, 2 ** 15), (2 ** 19 + 1, 2 ** 21)):
        assert call(M, R) == call(M, R, dd=None) == call(M, R, du=None) == mkq.MKQ_ERR_UNSUPPORTED, (M, R)
    for M, R in ((2 ** 20, 2 ** 20), (2 ** 26, 2 ** 14), (2 ** 14, 2 ** 22 - 1)):
        assert call(M, R) == mkq.MKQ_ERR_WORKSPACE, (M, R)
    assert call(2 ** 26, 2 ** 15, dd=None, du=None, dx=0x60000000000) == mkq.MKQ_ERR_WORKSPACE


def test_gradients_over_what_they_are_computed_from(lib):
    """The batch's rows, the hidden values and the other results are read or written beside the adapters' gradients."""
    M, K, N, rank, R = 100, 64, 96, 8, 3
    at = dict(dy=X, x=X + 0x1000000, hidden=X + 0x2000000, dx=X + 0x3000000, dd=X + 0x4000000, du=X + 0x5000000, steps=X + 0x6000000)
    size = dict(dy=2 * M * N, x=2 * M * K, hidden=4 * M * rank, dx=2 * M * K, dd=4 * R * rank * K, du=4 * R * rank * N, steps=4 * M)
    need = lib.mkq_low_rank_adapters_gradient_workspace_bytes(M, K, N, rank, R)

    def call(**kw):
        a = dict(at, **kw)
        v = lambda name: C.c_void_p(a[name]) if a[name] else None  # noqa: E731
        kept = a.get("kept", False)
        return lib.mkq_low_rank_adapters_gradient(v("dy"), F16, N, v("x"), mkq.MKQ_I8 if kept else F16, K, v("steps"), 64, P, v("hidden"), M, K, N, rank, R, P, P, F16, None,
                                                  None, 0, v("dx"), F16, K, v("dd"), v("du"), F32, 0, P, need, None)
    for result in ("dd", "du"):
        for other in ("dy", "x", "hidden", "dx", "du" if result == "dd" else "dd"):
            for to in (at[other], at[other] + size[other] - 16, at[other] - size[result] + 16):
                assert call(**{result: to}) == mkq.MKQ_ERR_UNSUPPORTED, (result, other, hex(to))
        assert call(kept=True, **{result: at["steps"] + size["steps"] - 16}) == mkq.MKQ_ERR_UNSUPPORTED
    for to in (at["hidden"], at["hidden"] + size["hidden"] - 16, at["hidden"] - size["dx"] + 16):
        assert call(dx=to) == mkq.MKQ_ERR_UNSUPPORTED
    # what is not read or written does not count
    assert call(dx=None, dd=None, hidden=None, du=at["dy"] + 16) == mkq.MKQ_ERR_NULL
    assert call(dd=None, du=at["dy"]) == call(du=None, dd=at["x"]) == mkq.MKQ_ERR_UNSUPPORTED
