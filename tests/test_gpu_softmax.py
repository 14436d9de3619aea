"""adacomp_bias_softmax and its backward pass against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import block64 as O
from paper_1712_02679_b200 import binding as B
from tests.block_util import DEV, ROUND, TINY, U, guarded, rng_state, to64, to_dev, within

pytestmark = pytest.mark.gpu
SEED, STEP, SITE = 55555555555, 2, 9


class Case:
    def __init__(self, b, h, q, k, kind="f32", causal=False, lens=None, p=0.0, buckets=(32, 128), both=True, q_offset=None,
                 scale=0.5, spread=3.0, pad=0, scores=None):
        r = np.random.default_rng(b * 1000003 + h * 10007 + q * 101 + k)
        self.dims, self.kind, self.causal, self.p, self.scale = (b, h, q, k), kind, causal, p, scale
        self.q_offset = k - q if q_offset is None else q_offset
        self.ld = k + pad
        s = r.normal(0, spread, (b, h, q, k)) if scores is None else scores
        self.scores = self.strided(to_dev(s, kind))
        self.dprobs = self.strided(to_dev(r.normal(0, 0.2, (b, h, q, k)), kind))
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.plan = B.adacomp_relpos_plan(buckets[0], buckets[1], both) if buckets else None
        self.table = to_dev(r.normal(0, 1, (buckets[0], h))) if buckets else None
        self.ids = O.buckets(q, k, self.q_offset, buckets[0], buckets[1], both) if buckets else None
        self.n = buckets[0] if buckets else 0
        self.rng = rng_state(SEED, STEP)
        self.fac = O.dropout_factors(b * h * q, k, p, SEED, STEP, SITE).reshape(b, h, q, k) if p else None
        self.keep = np.broadcast_to(O.kept(b, q, k, causal, self.q_offset, lens), (b, h, q, k))
        self.kw = dict(scale=scale, causal=causal, q_offset=self.q_offset, key_len=self.lens, p=p, rng=self.rng, site=SITE)

    def strided(self, t):
        """The same values in rows `ld` apart, NaN between them."""
        b, h, q, k = self.dims
        whole = torch.full((b, h, q, self.ld), float("nan"), dtype=t.dtype, device=DEV)
        whole[..., :k] = t
        return whole[..., :k]

    def output(self):
        b, h, q, k = self.dims
        whole, intact = guarded((b, h, q, self.ld), self.kind)
        return whole[..., :k], lambda: intact() and bool((whole[..., k:] == 7.0).all())

    def bias(self):
        return None if self.table is None else to64(self.table).T[:, self.ids]

    def oracle(self):
        return O.softmax(to64(self.scores), self.bias(), self.scale, self.keep)

    def reach(self):
        """Bound of |logit| over a row's kept finite entries, with the row's maximum: what exponents' errors scale with."""
        t = np.abs(np.where(self.keep, np.nan_to_num(to64(self.scores), nan=0, posinf=0, neginf=0), 0)) * abs(self.scale)
        if self.table is not None:
            t = t + np.abs(self.bias())
        return 2 * t.max(-1, keepdims=True, initial=0.0) + 1

    def forward(self):
        b, h, q, _ = self.dims
        probs, ok = self.output()
        lse, ok2 = guarded((b, h, q), "f32")
        B.adacomp_bias_softmax(self.scores, self.table, self.plan, probs, lse, **self.kw)
        assert ok() and ok2(), "wrote beside an output"
        return probs, lse

    def check_forward(self):
        probs, lse = self.forward()
        want, wlse = self.oracle()
        # a logit is off by a few roundings of its terms, a power by 2 more units, a row's sum by 128 (32 values a thread,
        # 5 + 5 exchanges, 8 CTAs), the division and the factor by 4
        rel = U * (16 * self.reach() + 160)
        wdrop = O.dropped(want, self.fac)
        within(to64(probs), wdrop, np.abs(wdrop) * (ROUND[self.kind] + rel) + TINY[self.kind] * 2, "probs")
        assert np.all(to64(probs)[~self.keep] == 0)
        within(to64(lse), wlse, rel[..., 0] + 2 * U * np.abs(np.where(np.isfinite(wlse), wlse, 0)), "lse")

    def backward(self, lse, table_grad=True):
        b, h, q, k = self.dims
        ds, ok = self.output()
        dt = ws = None
        ok2 = ok3 = lambda: True                                            # noqa: E731
        if self.table is not None and table_grad:
            dt, ok2 = guarded(self.table.shape, "f32")
            ws, ok3 = guarded((B.adacomp_bias_softmax_workspace(b, h, q, k, self.plan) // 4,), "f32", fill=-3.0)
            ws = ws.view(torch.uint8)
        B.adacomp_bias_softmax_backward(self.dprobs, self.scores, self.table, self.plan, lse, ds, dt, ws, **self.kw)
        assert ok() and ok2() and ok3(), "wrote beside an output"
        return ds, dt

    def check_backward(self):
        want, wlse = self.oracle()
        lse = to_dev(wlse)
        # (the row's statistic is an input: the definition is taken about the rounded one)
        finite = np.isfinite(wlse)
        shift = np.where(finite, wlse, 0.0) - np.where(finite, to64(lse), 0.0)
        probs = want * np.exp(shift)[..., None]
        wds, wdt = O.softmax_backward(to64(self.dprobs), probs, self.fac, self.scale, self.ids, self.n)
        ds, dt = self.backward(lse)
        dp = np.abs(O.dropped(to64(self.dprobs), self.fac))
        dp = np.where(self.keep, np.nan_to_num(dp, nan=0), 0)
        size = probs * (dp + (probs * dp).sum(-1, keepdims=True))
        rel = U * (16 * (self.reach() + np.abs(np.where(np.isfinite(wlse), wlse, 0))[..., None]) + 160)
        within(to64(ds), wds, np.abs(wds) * ROUND[self.kind] + abs(self.scale) * rel * size + TINY[self.kind] * 2, "dscores")
        assert np.all(to64(ds)[~self.keep] == 0)
        if dt is not None:
            # a chain of additions: 64 rows of 32 values in a thread at most, then exchanges, buckets and groups
            q, k = self.dims[2:]
            depth = min(q, 64) * 32 + 300
            off = (size * (rel + depth * U)).sum(0)
            bound = np.stack([np.where(self.ids == n, off, 0).sum((1, 2)) for n in range(self.n)])
            within(to64(dt), wdt, bound + np.abs(wdt) * U + 1e-30, "dtable")
            ds2, _ = self.backward(lse, table_grad=False)
            assert torch.equal(ds2, ds)
            _, dt2 = self.backward(lse)
            assert torch.equal(dt2, dt)
        return ds, dt


SHAPES = [(1, 1, 1, 1), (2, 3, 4, 8), (1, 2, 5, 7), (2, 2, 33, 33), (1, 3, 64, 255), (1, 2, 100, 256), (2, 1, 31, 300),
          (1, 2, 40, 512), (1, 1, 65, 777), (1, 1, 40, 1000), (1, 2, 30, 1024), (1, 1, 9, 1025), (1, 2, 8, 2048),
          (1, 1, 5, 4097), (1, 1, 3, 16384), (1, 1, 2, 16385), (1, 1, 3, 40000), (3, 70, 1, 90), (300, 4, 3, 64)]


@pytest.mark.parametrize("b,h,q,k", SHAPES)
@pytest.mark.parametrize("kind,causal,both,p,ragged", [("f32", False, True, 0.0, False), ("bf16", True, False, 0.1, False),
                                                        ("f16", False, True, 0.3, True), ("bf16", True, True, 0.0, True)])
def test_matches_definition(b, h, q, k, kind, causal, both, p, ragged):
    lens = None
    if ragged:
        lens = [int(v) for v in np.random.default_rng(k).integers(0, k + 1, b)]
    c = Case(b, h, q, k, kind, causal, lens, p, both=both)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("k", [70000, 70001, 131072])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_longest_rows(k, kind):
    c = Case(1, 1, 2, k, kind, True, [k - 1000], 0.1)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("b,h,q,k", [(1, 2, 130, 1024), (2, 2, 200, 997), (1, 1, 300, 1500), (1, 1, 90, 3001), (2, 1, 70, 4096)])
@pytest.mark.parametrize("kind,causal,scale", [("bf16", True, -0.5), ("f32", False, 0.0), ("f16", True, 0.25), ("f32", True, 1.0)])
def test_many_rows_and_scales(b, h, q, k, kind, causal, scale):
    lens = None if causal else [k - 300] * b
    c = Case(b, h, q, k, kind, causal, lens, 0.1, both=not causal, scale=scale)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("k,pad", [(40, 8), (1000, 24), (37, 3), (61, 4), (2000, 0), (2001, 7), (33, 7)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_spaced_apart(k, pad, kind):
    c = Case(2, 2, 11, k, kind, True, [k, k // 2], 0.2, pad=pad)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("buckets,both", [((2, 3), False), ((4, 2), True), ((16, 64), True), ((128, 1024), True),
                                           ((128, 1024), False), ((34, 18), True), (None, True)])
@pytest.mark.parametrize("q,k,q_offset", [(300, 300, 0), (50, 1500, 700), (70, 90, -40), (20, 64, 5000), (8, 2100, 30)])
def test_buckets_and_positions(buckets, both, q, k, q_offset):
    for causal in (False, True):
        c = Case(2, 2, q, k, "f32", causal, None, 0.0, buckets, both, q_offset)
        c.check_forward()
        c.check_backward()


def test_rows_that_keep_nothing_and_bad_values_in_masked_places():
    for k in (64, 65, 1500):
        for kind in ("f32", "bf16"):
            s = np.random.default_rng(k).normal(0, 1, (3, 2, 5, k))
            low = float(torch.finfo(torch.float32 if kind == "f32" else torch.bfloat16).min)
            s[0] = np.nan                                   # sequence of length 0
            s[1, :, :, 7:] = np.inf                         # beyond its length
            s[1, 0, 2, :7] = -np.inf                        # a row whose kept logits are all -inf
            s[2, 0, 1] = low                                # a row of the type's lowest value: uniform
            s[2, 0, 2, 5] = -np.inf                         # single entries masked by the caller
            s[2, 0, 3, 5:] = low
            c = Case(3, 2, 5, k, kind, False, [0, 7, k], 0.0, buckets=None, scale=1.0, scores=s)
            probs, lse = c.forward()
            want, wlse = c.oracle()
            rel = U * (16 * 30 + 160)                       # finite rows: |logit| < 5; the rows of `low` have equal logits
            within(to64(probs), want, np.abs(want) * (ROUND[kind] + rel) + 1e-30, "probs")
            assert np.all(to64(probs[0]) == 0) and np.all(np.isneginf(to64(lse[0])))
            assert np.all(to64(probs[1, 0, 2]) == 0) and np.isneginf(float(lse[1, 0, 2]))
            within(to64(probs[2, 0, 1]), np.full(k, 1 / k), (ROUND[kind] + rel) / k)
            c.dprobs[0] = float("nan")
            c.dprobs[1, :, :, 7:] = float("inf")
            ds, _ = c.backward(lse)
            got = to64(ds)
            assert np.all(got[0] == 0) and np.all(got[1, :, :, 7:] == 0) and np.all(got[1, 0, 2] == 0)
            assert np.all(np.isfinite(got[1]))
            wds, _ = O.softmax_backward(to64(c.dprobs), want, None, 1.0, None, 0)
            size = np.abs(to64(c.dprobs[2])).max()
            within(got[2], wds[2], np.abs(wds[2]) * ROUND[kind] + 2 * rel * want[2] * size + TINY[kind] * 2, "dscores")


def test_non_finite_rows_stay_their_own():
    s = np.random.default_rng(0).normal(0, 1, (1, 1, 6, 200))
    s[0, 0, 1, 3] = np.nan
    s[0, 0, 4, 150] = np.inf
    c = Case(1, 1, 6, 200, "f32", scores=s)
    probs, lse = c.forward()
    want, _ = c.oracle()
    bad = np.isnan(want).any(-1)
    assert bad[0, 0].tolist() == [False, True, False, False, True, False]
    got = to64(probs)
    assert np.array_equal(np.isnan(got).any(-1), bad)
    within(got[~bad], want[~bad], 2.0 ** -14)


@pytest.mark.parametrize("k", [128, 129, 3000])
def test_in_place_and_without_statistics(k):
    c = Case(2, 2, 9, k, "bf16", True, None, 0.2)
    probs, lse = c.forward()
    x = c.scores.clone()
    B.adacomp_bias_softmax(x, c.table, c.plan, x, None, **c.kw)
    assert torch.equal(x, probs)
    ds, _ = c.backward(lse)
    g = c.dprobs.clone()
    B.adacomp_bias_softmax_backward(g, c.scores, c.table, c.plan, lse, g, **c.kw)
    assert torch.equal(g, ds)
    s = c.scores.clone()
    B.adacomp_bias_softmax_backward(c.dprobs, s, c.table, c.plan, lse, s, **c.kw)
    assert torch.equal(s, ds)


def test_empty_sizes():
    plan = B.adacomp_relpos_plan(32, 128)
    table = torch.ones(32, 2, device=DEV)
    for shape in [(0, 2, 3, 4), (2, 2, 0, 4), (2, 2, 3, 0)]:
        t = torch.empty(shape, device=DEV)
        lse = torch.full(shape[:3], 5.0, device=DEV)
        dt = torch.full_like(table, 3.0)
        ws = torch.empty(B.adacomp_bias_softmax_workspace(*shape, plan), dtype=torch.uint8, device=DEV)
        B.adacomp_bias_softmax(t, table, plan, t, lse)
        assert torch.all(lse == -float("inf"))
        B.adacomp_bias_softmax_backward(t, t, table, plan, lse, t, dt, ws)
        assert torch.all(dt == 0)


def test_gradient_against_differences():
    """Directional derivatives of the 64-bit forward pass against the kernels' gradients of binary32 inputs."""
    for k, causal in ((48, False), (51, True)):
        c = Case(2, 3, 20, k, "f32", causal, None, 0.25, (16, 24), not causal)
        _, lse = c.forward()
        ds, dt = c.backward(lse)
        s0, t0, dp = to64(c.scores), to64(c.table), to64(c.dprobs)

        def loss(s, t):
            probs, _ = O.softmax(s, t.T[:, c.ids], c.scale, c.keep)
            return (O.dropped(probs, c.fac) * dp).sum()

        r = np.random.default_rng(2)
        vs, vt, e = r.normal(0, 1, s0.shape), r.normal(0, 1, t0.shape), 1e-5
        # gradients good to 2^-15 of what is added up (reach ~ 20: 16 * 20 + 160 roundings, and the sums)
        for grad, v, want in ((ds, vs, (loss(s0 + e * vs, t0) - loss(s0 - e * vs, t0)) / (2 * e)),
                              (dt, vt, (loss(s0, t0 + e * vt) - loss(s0, t0 - e * vt)) / (2 * e))):
            assert abs((to64(grad) * v).sum() - want) <= 2.0 ** -15 * np.abs(to64(grad) * v).sum() + 1e-6


def test_offsets_beyond_32_bits():
    b, h, q, k = 1, 2, 16400, 131072                        # 4.3e9 elements; only the last rows are looked at
    s = torch.zeros(b, h, q, k, dtype=torch.bfloat16, device=DEV)
    s[0, 1, -1] = torch.arange(k, device=DEV).fmod(7).to(torch.bfloat16)
    want = torch.softmax(s[0, 1, -1].double(), 0).cpu().numpy()
    B.adacomp_bias_softmax(s, None, None, s)
    within(to64(s[0, 1, -1]), want, want * (ROUND["bf16"] + 2.0 ** -14))
    within(to64(s[0, 1, -2]), np.full(k, 1 / k), 2.0 ** -9 / k)
    del s
    torch.cuda.empty_cache()


def test_captured_in_a_graph_on_another_stream():
    c = Case(2, 2, 64, 200, "bf16", False, [200, 150], 0.1)
    probs, lse = c.forward()
    p2, l2 = torch.empty(c.dims, dtype=torch.bfloat16, device=DEV), torch.empty_like(lse)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.adacomp_bias_softmax(c.scores.contiguous(), c.table, c.plan, p2, l2, **c.kw)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p2, probs) and torch.equal(l2, lse)


def test_refusals_of_the_binding():
    t = torch.zeros(2, 2, 4, 8, device=DEV)
    plan, table = B.adacomp_relpos_plan(8, 16), torch.zeros(8, 2, device=DEV)
    for bad in [lambda: B.adacomp_bias_softmax(t.transpose(2, 3), table, plan, t),
                lambda: B.adacomp_bias_softmax(t, table, plan, t.half()),
                lambda: B.adacomp_bias_softmax(t, table, plan, t[:, :, :, :4]),
                lambda: B.adacomp_bias_softmax(t, table, None, t),
                lambda: B.adacomp_bias_softmax(t, table[:4], plan, t),
                lambda: B.adacomp_bias_softmax(t, table.half(), plan, t),
                lambda: B.adacomp_bias_softmax(t[0], None, None, t[0]),
                lambda: B.adacomp_bias_softmax(t, None, None, t, key_len=torch.zeros(3, dtype=torch.int32, device=DEV)),
                lambda: B.adacomp_bias_softmax(t.transpose(1, 2), None, None, t.transpose(1, 2))]:
        with pytest.raises(ValueError):
            bad()
