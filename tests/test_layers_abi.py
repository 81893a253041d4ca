"""The layers' C entry points without a GPU: what they refuse, before any device work."""
import ctypes
import os

import pytest

_b = pytest.importorskip("paper_2605_12683_amd._binding")
BAD, WS = _b.DEER_ERR_INVALID_ARG, _b.DEER_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_b.LIB_PATH):
        pytest.skip("libdeer.so is not built (run __graft_entry__.build())")
    return _b.load()


_mem = (ctypes.c_char * 4096)()
P = [ctypes.addressof(_mem) + 256 * i for i in range(16)]     # addresses that are never read


def _shape(**kw):
    s = dict(dtype=_b.DEER_F32, H=4, Hk=2, Dk=8, Dv=8, per_step=0, scale=1.0)
    s.update(kw)
    return _b.deer_linattn_shape(*s.values())


def _view(p, sb=64, st=32, sh=8):
    return _b.deer_view(p, sb, st, sh)


BAD_SHAPES = [dict(dtype=3), dict(dtype=-1), dict(H=0), dict(Hk=0), dict(H=3), dict(H=1), dict(Dk=0), dict(Dk=257),
              dict(Dv=0), dict(Dv=257), dict(scale=float("nan")), dict(scale=float("inf")), dict(H=1 << 21, Hk=1), dict(H=16385, Hk=1)]


@pytest.mark.parametrize("kw", BAD_SHAPES)
def test_shapes(lib, kw):
    s = _shape(**kw)
    views = [ctypes.byref(_view(p)) for p in P[:4]]
    for op in (_b.DEER_OP_SOLVE, _b.DEER_OP_ADJOINT):
        assert lib.deer_linattn_workspace_bytes(ctypes.byref(s), 2, 16, op) == 0
    assert lib.deer_linattn(ctypes.byref(s), 2, 16, *views[:3], P[4], None, None, P[5], None, P[6], 1 << 30, None) == BAD
    assert lib.deer_last_error()
    assert lib.deer_linattn_adjoint(ctypes.byref(s), 2, 16, *views[:3], P[4], None, None, views[3], None, P[5], P[6],
                                    P[7], None, None, P[8], 1 << 30, None) == BAD
    assert lib.deer_linattn_step(ctypes.byref(s), 2, *views[:3], P[4], None, P[5], P[6], None) == BAD


def test_sizes_and_queries(lib):
    s = _shape()
    for B, T in ((0, 4), (4, 0), (-1, 4), (1 << 19, 4), (1 << 10, 1 << 30), (1, (1 << 30) + 1)):
        assert lib.deer_linattn_workspace_bytes(ctypes.byref(s), B, T, _b.DEER_OP_SOLVE) == 0, (B, T)
    assert lib.deer_linattn_workspace_bytes(ctypes.byref(s), 2, 16, _b.DEER_OP_JACOBIAN) == 0
    assert lib.deer_linattn_workspace_bytes(None, 2, 16, _b.DEER_OP_SOLVE) == 0
    for op in (_b.DEER_OP_SOLVE, _b.DEER_OP_ADJOINT):
        for dtype in range(3):
            for T in (1, 64, 65, 5000, 1 << 20):
                assert lib.deer_linattn_workspace_bytes(ctypes.byref(_shape(dtype=dtype)), 2, T, op) > 0


def _forward(lib, s, q=0, k=1, v=2, ld=4, o=5, state0=None, state=None, ws=6, n=1 << 30):
    a = lambda i: None if i is None else P[i]  # noqa: E731
    vw = lambda i: None if i is None else ctypes.byref(i if isinstance(i, _b.deer_view) else _view(P[i]))  # noqa: E731
    return lib.deer_linattn(ctypes.byref(s) if s else None, 2, 16, vw(q), vw(k), vw(v), a(ld), None, a(state0), a(o),
                            a(state), a(ws), n, None)


def test_forward_arguments(lib):
    s = _shape()
    assert _forward(lib, None) == BAD
    for x in ("q", "k", "v", "ld", "o"):
        assert _forward(lib, s, **{x: None}) == BAD, x
    assert _forward(lib, s, q=_view(None)) == BAD
    for st in (dict(sb=-1), dict(st=-1), dict(sh=-8), dict(st=(1 << 22) + 1)):
        assert _forward(lib, s, v=_view(P[2], **st)) == BAD and b"stride" in lib.deer_last_error()
    for o in (0, 1, 2, 4, 7):
        assert _forward(lib, s, o=o, state0=7) == BAD and b"input" in lib.deer_last_error()
    for state in (0, 1, 2, 4, 5):
        assert _forward(lib, s, state=state) == BAD
    assert _forward(lib, s, ws=None) == WS
    assert _forward(lib, s, n=0) == WS


def test_adjoint_arguments(lib):
    s = _shape()
    need = lib.deer_linattn_workspace_bytes(ctypes.byref(s), 2, 16, _b.DEER_OP_ADJOINT)

    def call(out, g=3, ws=15, n=1 << 30, state0=13, gs=14):
        v = [ctypes.byref(_view(P[i])) for i in range(3)]
        gv = None if g is None else ctypes.byref(_view(P[g]))
        return lib.deer_linattn_adjoint(ctypes.byref(s), 2, 16, *v, P[4], None, P[state0], gv, P[gs],
                                        *(None if i is None else P[i] for i in out), None if ws is None else P[ws], n, None)

    assert call((5, 6, 7, 8, 9), g=None) == BAD
    for i in range(3):
        out = [5, 6, 7, 8, 9]
        out[i] = None
        assert call(out) == BAD
    for i in range(5):
        for alias in (0, 1, 2, 3, 4, 13, 14):
            out = [5, 6, 7, 8, 9]
            out[i] = alias
            assert call(out) == BAD, (i, alias)
        for j in range(i):
            out = [5, 6, 7, 8, 9]
            out[i] = out[j]
            assert call(out) == BAD, (i, j)
    assert call((5, 6, 7, 8, 9), ws=None) == WS
    assert call((5, 6, 7, 8, 9), n=need - 1) == WS


def test_step_arguments(lib):
    s = _shape()
    v = [ctypes.byref(_view(P[i])) for i in range(3)]
    assert lib.deer_linattn_step(ctypes.byref(s), 0, *v, P[4], None, P[5], P[6], None) == BAD
    for ld, state, o in ((None, 5, 6), (4, None, 6), (4, 5, None), (4, 5, 5), (4, 0, 6), (4, 5, 1), (4, 4, 6)):
        a = [None if i is None else P[i] for i in (ld, state, o)]
        assert lib.deer_linattn_step(ctypes.byref(s), 2, *v, a[0], None, a[1], a[2], None) == BAD, (ld, state, o)


def _norm(**kw):
    n = dict(dtype=_b.DEER_BF16, wtype=_b.DEER_F32, G=2, D=16, w=P[0], b=P[1], eps=1e-5)
    n.update(kw)
    return ctypes.byref(_b.deer_norm(*n.values()))


@pytest.mark.parametrize("kw,rows", [
    (dict(dtype=9), 4), (dict(wtype=_b.DEER_F16), 4), (dict(wtype=7), 4), (dict(G=0), 4), (dict(D=0), 4),
    (dict(D=65537), 4), (dict(G=1 << 12, D=1 << 13), 1 << 12), (dict(eps=-1e-9), 4), (dict(eps=float("nan")), 4),
    (dict(eps=float("inf")), 4), (dict(G=(1 << 20) + 1, D=1), (1 << 20) + 1), (dict(), 0), (dict(), -2), (dict(), 3)])
def test_norms(lib, kw, rows):
    n = _norm(**kw)
    assert lib.deer_layernorm_workspace_bytes(n, rows) == 0
    assert lib.deer_layernorm(n, rows, P[2], P[3], P[4], P[5], None) == BAD
    assert lib.deer_last_error()
    assert lib.deer_layernorm_adjoint(n, rows, P[2], P[3], P[4], P[5], P[6], P[7], P[8], P[9], 1 << 30, None) == BAD


def test_norm_arguments(lib):
    n = _norm()
    assert lib.deer_layernorm(None, 4, P[2], P[3], None, None, None) == BAD
    for x, y, m, r in ((None, 3, 4, 5), (2, None, 4, 5), (2, 2, 4, 5), (2, 0, 4, 5), (2, 1, 4, 5), (2, 3, 3, 5), (2, 3, 4, 4),
                       (2, 3, 4, 2), (2, 3, 0, 5)):
        a = [None if i is None else P[i] for i in (x, y, m, r)]
        assert lib.deer_layernorm(n, 4, *a, None) == BAD, (x, y, m, r)
    need = lib.deer_layernorm_workspace_bytes(n, 4)
    assert need > 0

    def call(x=2, g=3, m=4, r=5, dx=6, dw=7, db=8, ws=9, size=1 << 30):
        a = [None if i is None else P[i] for i in (x, g, m, r, dx, dw, db, ws)]
        return lib.deer_layernorm_adjoint(n, 4, *a, size, None)

    for kw in (dict(x=None), dict(g=None), dict(m=None), dict(r=None), dict(dx=2), dict(dx=3), dict(dw=4), dict(db=5),
               dict(dw=0), dict(db=7), dict(dw=6), dict(dx=8)):
        assert call(**kw) == BAD, kw
    assert call(ws=None) == WS and call(size=need - 1) == WS
