"""Which rows eviction keeps: the steps of its selection on the host, against a sort."""
import numpy as np
import pytest

from paper_2511_12201_amd import binding as ob


def keys_of(weights):
    """32-bit keys in the order of the weights, as rows that their position does not spare are ranked."""
    u = np.ascontiguousarray(weights, dtype=np.float32).view(np.uint32)
    return np.where(u >> 31 != 0, ~u, u | np.uint32(1 << 31)).astype(np.uint32)


def check(weights, keep):
    keys = keys_of(weights)
    want = np.zeros(len(keys), dtype=bool)
    want[np.argsort(-keys.astype(np.int64), kind="stable")[:keep]] = True
    np.testing.assert_array_equal(ob.debug_evict_stay(keys, keep), want)


def below(x):
    return np.nextafter(np.float32(x), np.float32(0))


# The upper 11 bits of a key change at an eighth or a quarter of a power of two: 0.4375, 0.5, 0.875, 1, 1.25, ..
BORDERS = [0.4375, 0.5, 0.875, 1.0, 1.25, 3.5, 64.0]


@pytest.mark.parametrize("border", BORDERS)
@pytest.mark.parametrize("low,close,high", [(200, 200, 200), (200, 200, 7792), (200, 100, 2000), (1, 127, 500), (1, 128, 1), (0, 300, 300)])
def test_cuts_just_below_a_border_of_the_bins(border, low, close, high):
    """Rows of one bin from its middle to its last key, and many on the first key of the bin above."""
    rng = np.random.default_rng(low + close + high)
    w = np.concatenate([np.full(low, border * 0.97), np.full(close, below(border)), np.full(high, border)]).astype(np.float32)
    w = w[rng.permutation(len(w))]
    for keep in {high - 1, high, high + 1, high + close // 2, high + close - 1, high + close, high + close + 1, high + close + low // 2}:
        if 0 < keep < len(w):
            check(w, keep)


@pytest.mark.parametrize("border", BORDERS)
@pytest.mark.parametrize("spread", [1e-2, 1e-3, 1e-4, 1e-5, 3e-7])
@pytest.mark.parametrize("n", [300, 2000, 16384])
def test_cuts_among_weights_around_a_border(border, spread, n):
    rng = np.random.default_rng(n)
    for _ in range(4):
        w = (border * (1 + spread * rng.standard_normal(n))).astype(np.float32)
        above = int((w >= border).sum())
        for keep in [above + d for d in range(-4, 5)] + [1, n // 2, n - 1]:
            if 0 < keep < n:
                check(w, keep)


@pytest.mark.parametrize("seed", range(40))
def test_cuts_among_weights_of_many_shapes(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.choice([2, 100, 1000, 5000, 16384]))
    w = rng.choice([0.0, 1.0, -2.0]) + rng.choice([1e-6, 1e-3, 1.0, 1e6]) * (
        rng.standard_normal(n) if seed % 2 else np.exp(3 * rng.standard_normal(n)))
    w = np.where(rng.random(n) < rng.choice([0, 0.3, 0.9]), rng.choice(np.array([0.0, 1.0, np.inf, -np.inf])), w).astype(np.float32)
    for keep in {1, n // 3, n // 2, n - 1, *rng.integers(1, n, 6).tolist()}:
        if 0 < keep < n:
            check(w, keep)


def test_refusals():
    for keep in (0, 5, 6):
        with pytest.raises(ob.OmniError):
            ob.debug_evict_stay(np.arange(5, dtype=np.uint32), keep)
