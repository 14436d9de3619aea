"""Helpers of the block operators' GPU tests: types, and the bounds their results are held to."""
import numpy as np
import torch

DEV = torch.device("cuda:0")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, relative; and half the spacing of the smallest numbers
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
U = 2.0 ** -24


def to_dev(a, kind="f32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(DTYPES[kind])


def to64(t):
    return t.double().cpu().numpy()


def rng_state(seed, step):
    return torch.tensor([seed, step], dtype=torch.int64, device=DEV)


def within(got, want, bound, what=""):
    """Every element within its bound; non-finite values have to agree in kind."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), f"{what}: non-finite values differ"
    off = np.abs(np.where(odd, 0, got) - np.where(odd, 0, want))
    bad = ~(off <= np.broadcast_to(bound, off.shape)) & ~odd
    if bad.any():
        at = tuple(int(v) for v in np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {at}: got {got[at]!r}, want "
                             f"{want[at]!r}, bound {np.broadcast_to(bound, off.shape)[at]:.3e}")


def guarded(shape, kind, fill=7.0, pad=64):
    """A tensor in the middle of a larger buffer of a known value, and a check that the surroundings were not written."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * pad,), fill, dtype=DTYPES[kind], device=DEV)

    def intact():
        return bool((whole[:pad] == fill).all()) and bool((whole[pad + n:] == fill).all())

    return whole[pad:pad + n].view(shape), intact
