"""adacomp_dropout against the 64-bit definition: the mask bit for bit, values within one rounding."""
import numpy as np
import pytest
import torch

from oracle import block64 as O
from paper_1712_02679_b200 import binding as B
from tests.block_util import DEV, DTYPES, ROUND, TINY, U, guarded, rng_state, to64, to_dev, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 16), (17, 33), (1, 100003), (257, 1001), (300, 2048),
                                       (1025, 24), (2, 65537), (4099, 3)])
def test_matches_definition(rows, cols, kind):
    r = np.random.default_rng(rows * 7 + cols)
    x = to_dev(r.normal(0, 1, (rows, cols)), kind)
    seed, step, site, p = int(r.integers(0, 2 ** 62)), int(r.integers(0, 2 ** 40)), int(r.integers(0, 2 ** 32)), 0.3
    y, intact = guarded((rows, cols), kind)
    B.adacomp_dropout(x, y, p, rng_state(seed, step), site)
    f = O.dropout_factors(rows, cols, p, seed, step, site)
    want = O.dropped(to64(x), f)
    got = to64(y)
    assert np.array_equal(got == 0, want == 0)
    # the factor rounded, the product rounded, and the result rounded to its type
    within(got, want, np.abs(want) * (ROUND[kind] + 3 * U) + TINY[kind])
    assert intact()


@pytest.mark.parametrize("cols", [64, 65])
@pytest.mark.parametrize("p", [0.0, 1e-9, 2.0 ** -16, 0.5, 1.0 - 2.0 ** -16, 1.0])
def test_extreme_probabilities_and_non_finite_inputs(p, cols):
    x = torch.ones(64, cols, device=DEV)
    x[::2] = float("inf")
    x[1::4] = float("nan")
    y = torch.empty_like(x)
    B.adacomp_dropout(x, y, p, rng_state(11, 0), 1)
    f = O.dropout_factors(64, cols, p, 11, 0, 1)
    want = np.where(f == 0, 0.0, to64(x) * np.where(f == 0, 1.0, f))
    within(to64(y), want, np.abs(np.where(np.isfinite(want), want, 0)) * 4 * U)


@pytest.mark.parametrize("cols", [256, 255])
def test_in_place_backward_and_empty(cols):
    r = np.random.default_rng(3)
    x = to_dev(r.normal(0, 1, (100, cols)), "bf16")
    state = rng_state(5, 9)
    y = torch.empty_like(x)
    B.adacomp_dropout(x, y, 0.4, state, 2)
    z = x.clone()
    B.adacomp_dropout(z, z, 0.4, state, 2)
    assert torch.equal(y, z)
    ones = torch.ones_like(x)
    B.adacomp_dropout(ones, ones, 0.4, state, 2)            # the backward pass: same mask
    assert torch.equal(ones == 0, y == 0)
    empty = torch.empty(0, cols, device=DEV)
    B.adacomp_dropout(empty, empty, 0.4, state, 2)
    B.adacomp_dropout(empty.view(cols, 0), empty.view(cols, 0), 0.4, state, 2)


def test_another_stream_and_a_graph_that_draws_anew():
    x = torch.ones(64, 512, device=DEV)
    y = torch.empty_like(x)
    state = rng_state(77, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.adacomp_dropout(x, y, 0.5, state, 0)
    B.adacomp_dropout(x, y, 0.5, state, 0, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.adacomp_dropout(x, y, 0.5, state, 0)
        state[1] += 1
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(to64(y), O.dropout_factors(64, 512, 0.5, 77, step, 0))


@pytest.mark.parametrize("cols", [1 << 16, (1 << 16) + 1])
def test_offsets_beyond_32_bits(cols):
    rows = (1 << 16) + 8                                    # more than 2^32 elements
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    B.adacomp_dropout(x, x, 0.5, rng_state(8, 8), 0)
    w = O.philox([np.arange(-(-cols // 8)), np.full(-(-cols // 8), rows - 1), 8, 0], (8, 0))
    bits = np.stack([(v >> np.uint64(s)) & np.uint64(0xFFFF) for v in w for s in (0, 16)], -1).reshape(-1)[:cols]
    assert np.array_equal(to64(x[-1]), np.where(bits >= 32768, 2.0, 0.0))
    del x
    torch.cuda.empty_cache()


def test_refusals_of_the_binding():
    x = torch.zeros(8, 8, device=DEV)
    state = rng_state(0, 0)
    for bad in [lambda: B.adacomp_dropout(x.t(), x, 0.5, state), lambda: B.adacomp_dropout(x, x[:4], 0.5, state),
                lambda: B.adacomp_dropout(x, x.half(), 0.5, state), lambda: B.adacomp_dropout(x.int(), x.int(), 0.5, state),
                lambda: B.adacomp_dropout(x, x, 0.5, state.int()), lambda: B.adacomp_dropout(x, x, 0.5, state[:1])]:
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.AdaCompError):
        B.adacomp_dropout(x.view(-1)[1:9], x.view(-1)[1:9], 0.5, state)
    assert DTYPES
