"""adacomp_layer_norm and its backward pass against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import block64 as O
from paper_1712_02679_b200 import binding as B
from tests.block_util import DEV, DTYPES, ROUND, TINY, U, guarded, rng_state, to64, to_dev, within

pytestmark = pytest.mark.gpu
EPS = 1e-5
SEED, STEP, SITE = 987654321987, 5, 3


def _case(rows, cols, kind, param, fused, p, affine=True, offset=0.5):
    r = np.random.default_rng(rows * 131 + cols)
    s = {"x": to_dev(r.normal(offset, 1, (rows, cols)), kind),
         "res": to_dev(r.normal(0, 2, (rows, cols)), kind) if fused else None,
         "w": to_dev(r.normal(1, 0.3, cols), param) if affine else None,
         "b": to_dev(r.normal(0, 0.3, cols), param) if affine else None,
         "fac": O.dropout_factors(rows, cols, p, SEED, STEP, SITE) if p else None, "p": p, "rng": rng_state(SEED, STEP)}
    return s


def _n(t):
    return None if t is None else to64(t)


def _forward(s, kind):
    x = s["x"]
    y, ok_y = guarded(x.shape, kind)
    h, ok_h = guarded(x.shape, kind)
    mean, ok_m = guarded(x.shape[:1], "f32")
    rstd, ok_r = guarded(x.shape[:1], "f32")
    B.adacomp_layer_norm(x, s["w"], s["b"], y, mean, rstd, EPS, s["res"], h, s["p"], s["rng"], SITE)
    assert ok_y() and ok_h() and ok_m() and ok_r()
    return y, h, mean, rstd


def _check_forward(s, kind):
    y, h, mean, rstd = _forward(s, kind)
    wy, wh, wm, wr = O.layer_norm(_n(s["x"]), _n(s["res"]), _n(s["w"]), _n(s["b"]), EPS, s["fac"])
    # h: factor, product and sum in 32 bits, then its type's rounding
    big = np.abs(wh).max(1)
    terms = np.abs(wh) + (0 if s["res"] is None else 2 * np.abs(_n(s["res"])))
    eh = 4 * U * terms
    within(to64(h), wh, np.abs(wh) * ROUND[kind] + eh + TINY[kind], "h")
    # sums of a row: at most 64 roundings deep (16 values per thread, 5 + 5 exchanges, 8 CTAs, merging), each relative to
    # the row's largest value; var is a mean of squares, so rstd moves by half its relative error
    top = big + 4 * U * terms.max(1)
    within(to64(mean), wm, 64 * U * top, "mean")
    spread = 1 / wr
    er = 96 * U + 64 * U * top / spread * 2
    within(to64(rstd), wr, wr * er, "rstd")
    aw = 1.0 if s["w"] is None else np.abs(_n(s["w"]))
    ab = 0.0 if s["b"] is None else np.abs(_n(s["b"]))
    xhat = np.abs((wh - wm[:, None]) * wr[:, None])
    e32 = aw * (xhat * (er + 4 * U)[:, None] + ((64 * U * top)[:, None] + eh) * wr[:, None]) + 2 * U * (aw * xhat + ab)
    within(to64(y), wy, np.abs(wy) * ROUND[kind] + e32 + TINY[kind], "y")


def _check_backward(s, kind, param, with_dh):
    rows, cols = s["x"].shape
    r = np.random.default_rng(cols)
    h = s["x"]
    _, _, mean, rstd = O.layer_norm(_n(h), None, None, None, EPS)
    mean_d, rstd_d = to_dev(mean), to_dev(rstd)
    mean, rstd = to64(mean_d), to64(rstd_d)
    dy = to_dev(r.normal(0, 0.1, (rows, cols)), kind)
    dh = to_dev(r.normal(0, 0.1, (rows, cols)), kind) if with_dh else None
    dx, ok1 = guarded((rows, cols), kind)
    dr, ok2 = guarded((rows, cols), kind)
    dw, ok3 = guarded((cols,), param)
    db, ok4 = guarded((cols,), param)
    ws, ok5 = guarded((B.adacomp_layer_norm_workspace(rows, cols) // 4,), "f32", -3.0)
    ws = ws.view(torch.uint8)
    args = (dy, h, s["w"], mean_d, rstd_d, dx, dw, db, ws, dh, dr, s["p"], s["rng"], SITE)
    B.adacomp_layer_norm_backward(*args)
    assert ok1() and ok2() and ok3() and ok4() and ok5()
    wx, wr_, ww, wb = O.layer_norm_backward(_n(dy), _n(dh), _n(h), _n(s["w"]), mean, rstd, s["fac"])
    # xhat is off by a few roundings of h and mean times rstd; the row's sums are at most 64 roundings deep
    ndy = np.abs(_n(dy))
    exh = 4 * U * (np.abs(_n(h)) + np.abs(mean)[:, None]) * rstd[:, None]
    xhat = np.abs((_n(h) - mean[:, None]) * rstd[:, None])
    g = ndy * (1.0 if s["w"] is None else np.abs(_n(s["w"])))
    m1, m2 = g.mean(1, keepdims=True), (g * xhat).mean(1, keepdims=True)
    e = rstd[:, None] * (8 * U * g + 72 * U * m1 + 72 * U * xhat * m2 + exh * m2 + xhat * (g * exh).mean(1, keepdims=True))
    e += 2 * U * (np.abs(wr_) + (np.abs(_n(dh)) if dh is not None else 0))
    within(to64(dr), wr_, np.abs(wr_) * ROUND[kind] + e + TINY[kind], "dresidual")
    scale = 1.0 if s["fac"] is None else s["fac"]
    within(to64(dx), wx, np.abs(wx) * (ROUND[kind] + 3 * U) + e * scale + TINY[kind], "dx")
    # sums over rows: the rows of a thread, the CTA's groups (<= 16), the lines (<= 296 in 16 warps, then 16)
    depth = rows / 296 + 16 + 19 + 16 + 8
    within(to64(dw), ww, np.abs(ww) * ROUND[param] + (ndy * (depth * U * xhat + exh)).sum(0) + TINY[param], "dweight")
    within(to64(db), wb, np.abs(wb) * ROUND[param] + depth * U * ndy.sum(0) + TINY[param], "dbias")
    # the same bytes again, and without the optional outputs
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    B.adacomp_layer_norm_backward(dy, h, s["w"], mean_d, rstd_d, dx2, dw2, None, ws, dh, None, s["p"], s["rng"], SITE)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)


SHAPES = [(1, 1), (3, 7), (2, 8), (70, 64), (33, 100), (129, 255), (40, 256), (65, 1000), (17, 1001), (301, 1024), (9, 2056),
          (5, 4095), (6, 4096), (4, 4104), (3, 8191), (3, 8192), (2, 8200), (3, 16384), (2, 20001), (2, 65536), (1, 65535),
          (2500, 96)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind,param,fused,p", [("f32", "f32", False, 0.0), ("bf16", "f32", True, 0.1),
                                                 ("f16", "f16", True, 0.0), ("bf16", "bf16", False, 0.25)])
def test_matches_definition(rows, cols, kind, param, fused, p):
    s = _case(rows, cols, kind, param, fused, p)
    _check_forward(s, kind)
    _check_backward(s, kind, param, fused)


# enough rows for the kernels that give a thread several blocks of eight columns
@pytest.mark.parametrize("rows,cols", [(1300, 264), (1203, 300), (1250, 512), (1190, 777), (1200, 1024), (1185, 1001),
                                       (700, 2056), (650, 2047), (320, 4096), (400, 4100), (160, 8200), (150, 16387)])
@pytest.mark.parametrize("kind,param,fused,p", [("f32", "f32", True, 0.1), ("bf16", "f32", True, 0.1),
                                                 ("f16", "f16", False, 0.0)])
def test_many_rows(rows, cols, kind, param, fused, p):
    s = _case(rows, cols, kind, param, fused, p)
    _check_forward(s, kind)
    _check_backward(s, kind, param, fused)


@pytest.mark.parametrize("cols", [64, 1001, 4096])
def test_without_parameters_and_with_a_large_mean(cols):
    s = _case(12, cols, "f32", "f32", True, 0.1, affine=False, offset=1000.0)
    _check_forward(s, "f32")
    _check_backward(s, "f32", "f32", True)


@pytest.mark.parametrize("cols", [128, 129, 9000])
def test_in_place(cols):
    s = _case(20, cols, "bf16", "f32", True, 0.2)
    y, h, mean, rstd = _forward(s, "bf16")
    x, res = s["x"].clone(), s["res"].clone()
    B.adacomp_layer_norm(x, s["w"], s["b"], x, None, None, EPS, res, res, 0.2, s["rng"], SITE)
    assert torch.equal(x, y) and torch.equal(res, h)
    dy, dh = torch.randn_like(y), torch.randn_like(y)
    dx, dr = torch.empty_like(y), torch.empty_like(y)
    B.adacomp_layer_norm_backward(dy, h, s["w"], mean, rstd, dx, dh_in=dh, dresidual=dr, p=0.2, rng=s["rng"], site=SITE)
    B.adacomp_layer_norm_backward(dy, h, s["w"], mean, rstd, dy, dh_in=dh, dresidual=dh, p=0.2, rng=s["rng"], site=SITE)
    assert torch.equal(dy, dx) and torch.equal(dh, dr)


def test_rows_of_one_value_zero_rows_and_non_finite_rows():
    x = torch.full((4, 512), 3.0, device=DEV)
    x[2, 100] = float("nan")
    x[3, 7] = float("inf")
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    B.adacomp_layer_norm(x, None, None, y, mean, rstd, EPS)
    assert torch.all(y[:2] == 0) and torch.all(y[2:].isnan())          # a bad row stays its own
    within(to64(rstd[:2]), np.full(2, EPS ** -0.5), 4 * U * EPS ** -0.5)
    for cols in (512, 513):
        e = torch.empty(0, cols, device=DEV)
        st = torch.empty(0, device=DEV)
        w = torch.ones(cols, device=DEV)
        dw, db = torch.full_like(w, 9.0), torch.full_like(w, 9.0)
        ws = torch.empty(B.adacomp_layer_norm_workspace(0, cols), dtype=torch.uint8, device=DEV)
        B.adacomp_layer_norm(e, w, w, e, st, st)
        B.adacomp_layer_norm_backward(e, e, w, st, st, e, dw, db, ws)
        assert torch.all(dw == 0) and torch.all(db == 0)


@pytest.mark.parametrize("cols,p", [(40, 0.2), (41, 0.2), (1500, 0.0)])
def test_gradient_against_differences(cols, p):
    """Directional derivatives of the 64-bit forward pass against the kernels' gradients of binary32 inputs."""
    s = _case(6, cols, "f32", "f32", True, p)
    r = np.random.default_rng(1)
    dy, dh = r.normal(0, 1, (6, cols)).astype(np.float32), r.normal(0, 1, (6, cols)).astype(np.float32)
    _, h, mean, rstd = _forward(s, "f32")
    dx, dr, dw, db = (torch.empty_like(t) for t in (s["x"], s["x"], s["w"], s["b"]))
    ws = torch.empty(B.adacomp_layer_norm_workspace(6, cols), dtype=torch.uint8, device=DEV)
    B.adacomp_layer_norm_backward(to_dev(dy), h, s["w"], mean, rstd, dx, dw, db, ws, to_dev(dh), dr, p, s["rng"], SITE)
    base = {k: _n(s[k]) for k in ("x", "res", "w", "b")}

    def loss(**kw):
        a = {**base, **kw}
        y, hh, _, _ = O.layer_norm(a["x"], a["res"], a["w"], a["b"], EPS, s["fac"])
        return (y * dy).sum() + (hh * dh).sum()

    for key, grad in (("x", dx), ("res", dr), ("w", dw), ("b", db)):
        v = r.normal(0, 1, base[key].shape)
        want = (loss(**{key: base[key] + 1e-5 * v}) - loss(**{key: base[key] - 1e-5 * v})) / 2e-5
        # the kernels' gradients are good to 2^-17 of the terms added here (sums 64 roundings deep)
        assert abs((to64(grad) * v).sum() - want) <= 2.0 ** -17 * np.abs(to64(grad) * v).sum() + 1e-6


def test_captured_in_a_graph_on_another_stream():
    s = _case(50, 768, "bf16", "f32", True, 0.1)
    y, h, mean, rstd = _forward(s, "bf16")
    y2, h2 = torch.empty_like(y), torch.empty_like(h)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.adacomp_layer_norm(s["x"], s["w"], s["b"], y2, None, None, EPS, s["res"], h2, 0.1, s["rng"], SITE)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2)


def test_refusals_of_the_binding():
    x = torch.zeros(8, 64, device=DEV)
    w = torch.zeros(64, device=DEV)
    for bad in [lambda: B.adacomp_layer_norm(x, w[:32], None, x), lambda: B.adacomp_layer_norm(x, w, w.half(), x),
                lambda: B.adacomp_layer_norm(x.t(), None, None, x.t()), lambda: B.adacomp_layer_norm(x, w, w, x.half()),
                lambda: B.adacomp_layer_norm(x, w, w, x, torch.zeros(7, device=DEV)),
                lambda: B.adacomp_layer_norm(x.double(), None, None, x.double())]:
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.AdaCompError):
        B.adacomp_layer_norm(x, w.half(), None, x)               # binary16 parameters for binary32 activations
    assert DTYPES
