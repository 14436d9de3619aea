"""The differentiable functions against torch's derivatives of the same formulas in 64 bits, and a small block trained
through packed gradients."""
import math

import numpy as np
import pytest
import torch

from oracle import block64 as O
from paper_1712_02679_b200 import block, block_step
from tests.block_util import DEV

pytestmark = pytest.mark.gpu
SEED, SITE = 321, 4


def _factors(shape, p, step=0, site=SITE):
    f = O.dropout_factors(math.prod(shape[:-1]), shape[-1], p, SEED, step, site).reshape(shape)
    return torch.from_numpy(f).to(DEV)


def _agree(got, want, what):
    """Binary32 kernels against 64 bits: sums of a few hundred terms, each good to a few units."""
    scale = want.abs().max().clamp(min=1e-6)
    assert ((got.double() - want).abs().max() / scale).item() < 2.0 ** -16, what


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("cols", [64, 77])
def test_dropout_and_norms(p, cols):
    torch.manual_seed(cols)
    x, r = (torch.randn(3, 11, cols, device=DEV, requires_grad=True) for _ in range(2))
    w, b = (torch.randn(cols, device=DEV, requires_grad=True) for _ in range(2))
    u, v = torch.randn(2, 3, 11, cols, device=DEV).double()
    rng = block.Rng(SEED)
    y, h = block.add_layer_norm(x, r, w, b, p, rng, SITE)
    z = block.dropout(block.layer_norm(h, w, None), p, rng, SITE + 1)
    got = torch.autograd.grad((y.double() * u).sum() + (z.double() * v).sum(), (x, r, w, b))
    x6, r6, w6, b6 = (t.detach().double().requires_grad_() for t in (x, r, w, b))
    f1, f2 = (_factors(x.shape, p, site=s) if p else 1.0 for s in (SITE, SITE + 1))
    h6 = r6 + x6 * f1
    y6 = torch.nn.functional.layer_norm(h6, (cols,), w6, b6, 1e-5)
    z6 = torch.nn.functional.layer_norm(h6, (cols,), w6, None, 1e-5) * f2
    want = torch.autograd.grad((y6 * u).sum() + (z6 * v).sum(), (x6, r6, w6, b6))
    _agree(y, y6, "y")
    _agree(z, z6, "z")
    for g, t, name in zip(got, want, ("dx", "dresidual", "dweight", "dbias")):
        _agree(g, t, name)


@pytest.mark.parametrize("p,causal", [(0.0, True), (0.25, False)])
def test_bias_softmax(p, causal):
    torch.manual_seed(1)
    b, h, q, k = 2, 3, 9, 21
    s = torch.randn(b, h, q, k, device=DEV, requires_grad=True)
    plan = block.relpos(8, 12, bidirectional=not causal)
    table = torch.randn(8, h, device=DEV, requires_grad=True)
    lens = torch.tensor([21, 15], dtype=torch.int32, device=DEV)
    u = torch.randn(b, h, q, k, device=DEV).double()
    rng = block.Rng(SEED)
    y = block.bias_softmax(s, table, plan, 0.7, causal, None, lens, p, rng, SITE)
    got = torch.autograd.grad((y.double() * u).sum(), (s, table))
    s6, t6 = s.detach().double().requires_grad_(), table.detach().double().requires_grad_()
    ids = torch.from_numpy(O.buckets(q, k, k - q, 8, 12, not causal)).to(DEV)
    keep = torch.from_numpy(np.broadcast_to(O.kept(b, q, k, causal, k - q, [21, 15]), (b, h, q, k)).copy()).to(DEV)
    y6 = torch.softmax((s6 * 0.7 + t6.t()[:, ids]).masked_fill(~keep, -math.inf), -1)
    y6 = y6 * (_factors(s.shape, p) if p else 1.0)
    want = torch.autograd.grad((y6 * u).sum(), (s6, t6))
    _agree(y, y6, "probs")
    _agree(got[0], want[0], "dscores")
    _agree(got[1], want[1], "dtable")


def test_an_rng_that_moved_on_is_refused():
    x = torch.randn(4, 32, device=DEV, requires_grad=True)
    rng = block.Rng(5)
    y = block.dropout(x, 0.5, rng)
    rng.advance()
    with pytest.raises(RuntimeError, match="moved on"):
        y.sum().backward()
    with pytest.raises(ValueError):
        block.dropout(x, 0.5, None)


def test_training_through_packed_gradients_learns_the_task():
    """Chance is ln 24 = 3.18; a block that looks a word's length back reaches a small fraction of it."""
    losses = block_step.train(steps=300, k=2)
    assert all(math.isfinite(v) for v in losses)
    assert abs(losses[0] - math.log(block_step.VOCAB)) < 1.0
    assert np.mean(losses[-20:]) < 0.5 * losses[0], losses[::25]
