"""The 64-bit definitions the block operators are compared with: the generator's published vectors, gradients against
differences, and the buckets of the library's plan against the formula.  CPU only."""
import numpy as np
import pytest

from oracle import block64 as O
from paper_1712_02679_b200 import binding as B


def test_philox_published_vectors():
    """Known-answer vectors of Philox4x32-10 published with the generator."""
    f = 0xFFFFFFFF
    cases = [([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
             ([f, f, f, f], [f, f], [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
             ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
              [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]
    for counter, key, want in cases:
        assert [int(v) for v in O.philox(counter, key)] == want


@pytest.mark.parametrize("p", [0.1, 0.25, 0.5, 0.9])
def test_kept_fraction_and_mean(p):
    f = O.dropout_factors(512, 1000, p, 123456789012345, 7, 3)
    n, t = f.size, O.threshold(p) / 65536
    assert abs((f == 0).mean() - t) < 5 * np.sqrt(t * (1 - t) / n)
    assert abs(f.mean() - 1.0) < 5 * np.sqrt(t / (1 - t) / n)
    # rows, steps, sites and seeds draw different masks
    same = [(O.dropout_factors(512, 1000, p, *a) == f).mean() for a in
            [(123456789012346, 7, 3), (123456789012345, 8, 3), (123456789012345, 7, 4)]]
    agree = t * t + (1 - t) ** 2
    assert all(abs(s - agree) < 0.01 for s in same)
    assert abs((f[1:] == f[:-1]).mean() - agree) < 0.01


def test_extremes_of_p():
    assert np.all(O.dropout_factors(3, 17, 0.0, 5, 0, 0) == 1.0)
    assert np.all(O.dropout_factors(3, 17, 1.0, 5, 0, 0) == 0.0)


def _difference(f, x, v, h):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("cols,res,drop,affine", [(1, False, False, True), (7, True, True, True), (64, True, True, False),
                                                   (33, False, True, True)])
def test_layer_norm_gradient_against_differences(cols, res, drop, affine):
    rng = np.random.default_rng(cols)
    rows, eps = 5, 1e-5
    x, r, dy, dh = (rng.normal(0, 1, (rows, cols)) for _ in range(4))
    w, b = (rng.normal(1, 0.3, cols), rng.normal(0, 0.3, cols)) if affine else (None, None)
    r = r if res else None
    fac = O.dropout_factors(rows, cols, 0.3, 99, 1, 2) if drop else None

    def loss(x=x, r=r, w=w, b=b):
        y, h, _, _ = O.layer_norm(x, r, w, b, eps, fac)
        return (y * dy).sum() + (h * dh).sum()

    _, h, mean, rstd = O.layer_norm(x, r, w, b, eps, fac)
    dx, dr, dw, db = O.layer_norm_backward(dy, dh, h, w, mean, rstd, fac)
    # central differences of a smooth function: error O(step^2) of curvature ~ rstd^3, and 1e-16 / step of rounding
    step = 1e-6
    for value, grad, f in [(x, dx, lambda t: loss(x=t)), (r, dr, lambda t: loss(r=t)), (w, dw, lambda t: loss(w=t)),
                           (b, db, lambda t: loss(b=t))]:
        if value is None:
            continue
        v = rng.normal(0, 1, value.shape)
        got, want = (grad * v).sum(), _difference(f, value, v, step)
        assert abs(got - want) <= 1e-6 * max(1.0, np.abs(grad * v).sum())


@pytest.mark.parametrize("causal,both,lens", [(False, True, None), (True, False, None), (False, True, [0, 5]),
                                               (True, False, [9, 3])])
def test_softmax_gradient_against_differences(causal, both, lens):
    rng = np.random.default_rng(17)
    b, h, q, k, nb, far = 2, 3, 6, 9, 8, 16
    s, dpr = rng.normal(0, 2, (b, h, q, k)), rng.normal(0, 1, (b, h, q, k))
    table = rng.normal(0, 1, (nb, h))
    ids = O.buckets(q, k, k - q, nb, far, both)
    keep = O.kept(b, q, k, causal, k - q, lens)
    fac = O.dropout_factors(b * h * q, k, 0.25, 4242, 3, 1).reshape(b, h, q, k)

    def loss(s=s, table=table):
        probs, _ = O.softmax(s, table.T[:, ids], 0.5, keep)
        return (O.dropped(probs, fac) * dpr).sum()

    probs, _ = O.softmax(s, table.T[:, ids], 0.5, keep)
    ds, dtable = O.softmax_backward(dpr, probs, fac, 0.5, ids, nb)
    for value, grad, f in [(s, ds, lambda t: loss(s=t)), (table, dtable, lambda t: loss(table=t))]:
        v = rng.normal(0, 1, value.shape)
        assert abs((grad * v).sum() - _difference(f, value, v, 1e-6)) <= 1e-7 * max(1.0, np.abs(grad * v).sum())


@pytest.mark.parametrize("nb,far,both", [(32, 128, True), (32, 128, False), (16, 64, True), (64, 256, True), (2, 2, False),
                                         (4, 3, True), (128, 1024, True), (128, 1024, False), (10, 100, True), (34, 18, True)])
def test_plan_agrees_with_the_formula(nb, far, both):
    plan = B.adacomp_relpos_plan(nb, far, both)
    first = list(plan.first[:plan.side])
    assert plan.side == (nb // 2 if both else nb) and first[0] == 0 and first == sorted(first)
    for d in range(-far - 50, far + 51):
        away = abs(d) if both else max(-d, 0)
        got = max(k for k in range(plan.side) if first[k] <= away) + (plan.side if both and d > 0 else 0)
        assert got == O.bucket(d, nb, far, both), d


def test_rows_that_keep_nothing_are_zeros():
    s = np.array([[[[np.nan, np.inf, -np.inf]]], [[[-np.inf, -np.inf, 5.0]]]])
    probs, lse = O.softmax(s, None, 1.0, O.kept(2, 1, 3, False, 0, [0, 2]))
    assert np.all(probs == 0) and np.all(lse == -np.inf)
