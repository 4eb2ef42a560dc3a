"""Random sequences of the three block-cache calls against their definitions, whole arrays compared: fleet shapes, block sizes, pools
that run short, requests longer than a row, counts that cannot be, ragged new tokens and rooms that are too small."""
import numpy as np
import pytest

from paper_2605_06113_b200 import binding, build

from cache_reference import EMPTY, MOST
from test_gpu_cache import Pair, _walk

pytestmark = pytest.mark.gpu


def _shape(rng):
    while True:
        B = int(rng.choice([1, 2, 7, 8, 31, 32, 33, 40, 63, 64, 65, 96, 128, 129, 200, 256]))
        G, slots = int(rng.integers(1, 65)), int(10 ** rng.uniform(2, 4.2))
        N = max(1, slots // (G * B))
        t = int(rng.choice([1, 2, 3, 4, 5, 7, 8, 16, 24, 33, 64, 128, 1000]))
        T, P = int(10 ** rng.uniform(0, 3.3)), int(10 ** rng.uniform(0, 4))
        if N * G * (P + B * T) <= 6e6:
            return N, G, B, t, P, T


def _sequence(rng):
    N, G, B, t, P, T = _shape(rng)
    p = Pair(N, G, B, t, P, T, seed=int(rng.integers(1 << 30)))
    f = p.f
    n = np.zeros((N, G, B), np.int64)
    for _ in range(4):
        n = _walk(rng, f, n, rng.choice([0, 0.01, 0.3, 0.9]), rng.choice([0, 0.1, 0.6, 1.0]), int(rng.choice([0, 1, 1, 5, t, 3 * t])))
        if rng.random() < 0.2:                                    # requests longer than a row of the table
            n = np.where(rng.random(n.shape) < 0.1, T * t + rng.integers(0, 3 * t + 1, n.shape), n)
        step = rng.integers(-5, 10 ** 6, N).astype(np.int32) if rng.random() < 0.5 else None
        length = np.where(n > 0, n - (0 if step is None else step[:, None, None]), 0 if step is None else EMPTY).astype(np.int32)
        if rng.random() < 0.4:
            p.update(length, step, out=True)                      # looked at and dropped
        p.update(length, step)
        n_new = rng.integers(-2, int(rng.choice([2, 5, 60, 2000])), n.shape).astype(np.int32)
        if rng.random() < 0.5:
            n_new = np.where(rng.random(n.shape) < 0.9, 0, n_new).astype(np.int32)
        if np.minimum(np.maximum(n_new, 0), n).sum() < 1e5:
            p.slots(length, int(10 ** rng.uniform(0, 4.2)) + 1, n_new, step)
        p.slots(length, int(rng.integers(1, B + 3)), step=step)
        p.pages(length, step)
        if rng.random() < 0.1:                                    # a count that cannot be, or that hides blocks
            at, value = (int(rng.integers(N)), int(rng.integers(G))), int(rng.choice([-1, P + 1, MOST, -(2 ** 31), P]))
            f.n_free[at] = p.c.n_free[at] = value


@pytest.mark.parametrize("seed", range(10))
def test_random_sequences(seed):
    rng = np.random.default_rng(1000 + seed)
    for _ in range(8):
        _sequence(rng)


def test_random_sequences_on_the_range_checked_build():
    binding.use_library(build.build_debug())
    try:
        hits = binding.lib().br_debug_bounds_hits()
        assert hits >= 0
        rng = np.random.default_rng(2000)
        for _ in range(20):
            _sequence(rng)
        assert binding.lib().br_debug_bounds_hits() == hits
    finally:
        binding.use_library(None)
