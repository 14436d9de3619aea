"""What the block operators refuse, on the host and before any CUDA call.  CPU only."""
import ctypes as C

import pytest
import torch

from paper_1712_02679_b200 import binding as B, build

A = 0x1000          # fake, 16-byte aligned, never dereferenced: the checks come first
NULL, SHAPE, TYPE, VALUE, WORKSPACE, ALIGN = -1, -10, -11, -12, -13, -3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def test_error_texts():
    texts = {B.adacomp_strerror(c) for c in (SHAPE, TYPE, VALUE, WORKSPACE)}
    assert len(texts) == 4 and "unknown error code" not in texts


def test_dropout(lib):
    f = lib.adacomp_dropout

    def call(x=A, y=A, rows=4, cols=8, type=1, p=0.5, rng=A):
        return f(x, y, rows, cols, type, p, rng, 0, None)

    assert call(x=None) == call(y=None) == call(rng=None) == NULL
    assert call(type=3) == TYPE
    assert call(p=-0.1) == call(p=1.5) == call(p=float("nan")) == VALUE
    assert call(x=A + 2) == call(y=A + 8) == call(rng=A + 4) == ALIGN
    assert call(rows=1 << 32) == SHAPE
    assert call(x=None, rows=0) == call(x=None, cols=0) == 0


def _norm(**kw):
    d = dict(rows=4, cols=64, type=1, param_type=0, eps=1e-5, p=0.0, site=0, rng=None)
    d.update(kw)
    return C.byref(B.adacomp_norm_options(*d.values()))


def test_layer_norm(lib):
    def call(x=A, res=None, w=A, b=A, h=None, y=A, mean=A, rstd=A, opt=None, **kw):
        return lib.adacomp_layer_norm(x, res, w, b, h, y, mean, rstd, opt or _norm(**kw), None)

    def back(dy=A, dh=None, h=A, w=A, mean=A, rstd=A, dx=A, dr=None, dw=A, db=A, ws=A, nbytes=1 << 30, **kw):
        return lib.adacomp_layer_norm_backward(dy, dh, h, w, mean, rstd, dx, dr, dw, db, ws, nbytes, _norm(**kw), None)

    for f in (call, back):
        assert f(cols=0) == f(cols=65537) == f(rows=1 << 32) == SHAPE
        assert f(type=3) == f(param_type=7) == f(type=1, param_type=2) == TYPE
        assert f(eps=-1.0) == f(eps=float("inf")) == f(eps=float("nan")) == f(p=2.0) == VALUE
        assert f(p=0.5) == NULL and f(p=0.5, rng=A + 4) == ALIGN
        assert f(w=A + 4) == ALIGN
    assert call(x=None) == call(y=None) == NULL
    assert call(x=A + 8) == call(res=A + 2) == call(y=A + 1) == call(h=A + 4) == call(mean=A + 4) == ALIGN
    assert lib.adacomp_layer_norm(A, None, A, A, None, A, A, A, None, None) == NULL
    assert call(x=None, y=None, rows=0) == 0
    assert back(dy=None) == back(h=None) == back(mean=None) == back(rstd=None) == back(ws=None) == NULL
    assert back(dx=A + 8) == back(dr=A + 2) == back(dw=A + 4) == back(db=A + 4) == back(ws=A + 8) == back(dh=A + 8) == ALIGN
    need = B.adacomp_layer_norm_workspace(4, 64)
    assert need > 0 and back(nbytes=need - 1) == WORKSPACE
    assert B.adacomp_layer_norm_workspace(4, 0) == B.adacomp_layer_norm_workspace(4, 65537) == 0


def test_buckets(lib):
    for bad in [(0, 128, 1), (1, 128, 0), (3, 128, 1), (2, 128, 1), (130, 512, 1), (32, 8, 1), (32, 16, 0), (32, 1025, 1)]:
        with pytest.raises(B.AdaCompError) as e:
            B.adacomp_relpos_plan(*bad)
        assert e.value.code == SHAPE, bad
    assert lib.adacomp_relpos_plan(32, 128, 1, None) == NULL


def _soft(**kw):
    d = dict(batch=2, heads=3, q_len=4, k_len=8, ld=8, type=1, scale=1.0, causal=0, q_offset=0, key_len=None, p=0.0, site=0,
             rng=None)
    d.update(kw)
    return C.byref(B.adacomp_softmax_options(*d.values()))


def test_bias_softmax(lib):
    plan = B.adacomp_relpos_plan(32, 128)

    def call(s=A, table=A, rel=plan, probs=A, lse=A, **kw):
        return lib.adacomp_bias_softmax(s, table, rel if rel is None else C.byref(rel), probs, lse, _soft(**kw), None)

    def back(s=A, table=A, rel=plan, dp=A, lse=A, ds=A, dt=A, ws=A, nbytes=1 << 30, **kw):
        return lib.adacomp_bias_softmax_backward(dp, s, table, rel if rel is None else C.byref(rel), lse, ds, dt, ws, nbytes,
                                                 _soft(**kw), None)

    for f in (call, back):
        assert f(s=None) == f(rel=None) == f(p=0.1) == NULL
        assert f(type=3) == TYPE
        assert f(ld=7) == f(k_len=131073, ld=131073) == f(q_offset=1 << 30 | 1) == f(q_offset=-(1 << 30) - 1) == SHAPE
        assert f(q_len=1 << 30) == f(batch=1 << 16, heads=1 << 16) == f(batch=1 << 16, heads=1 << 10, q_len=64) == SHAPE
        assert f(scale=float("nan")) == f(scale=float("inf")) == f(p=-1.0) == VALUE
        assert f(s=A + 8) == f(lse=A + 4) == f(key_len=A + 2) == f(table=A + 2) == f(p=0.1, rng=A + 1) == ALIGN
    assert call(probs=None) == NULL and call(probs=A + 2) == ALIGN
    assert back(dp=None) == back(ds=None) == back(lse=None) == back(ws=None) == back(table=None) == NULL
    assert back(ds=A + 2) == back(dt=A + 4) == back(ws=A + 4) == back(dp=A + 8) == ALIGN
    need = B.adacomp_bias_softmax_workspace(2, 3, 4, 8, plan)
    assert need > 0 and back(nbytes=need - 1) == WORKSPACE
    assert lib.adacomp_bias_softmax(A, None, None, A, A, None, None) == NULL
    assert lib.adacomp_bias_softmax(None, None, None, None, None, _soft(batch=0), None) == 0
    for field, value in [("side", 1), ("num_buckets", 30), ("num_buckets", 256), ("max_distance", 2000)]:
        bad = B.adacomp_relpos_plan(32, 128)
        setattr(bad, field, value)
        assert call(rel=bad) == back(rel=bad) == SHAPE, field
    for at, value in [(0, 1), (3, 0), (15, 5000)]:
        bad = B.adacomp_relpos_plan(32, 128)
        bad.first[at] = value
        assert call(rel=bad) == back(rel=bad) == SHAPE, at


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 16)
    with pytest.raises(ValueError, match="CUDA"):
        B.adacomp_dropout(x, x, 0.5, None)
    with pytest.raises(ValueError, match="CUDA"):
        B.adacomp_layer_norm(x, None, None, x)
    s = torch.zeros(1, 1, 4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        B.adacomp_bias_softmax(s, None, None, s)
