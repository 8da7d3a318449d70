"""Which coefficients the orthogonalised updates accept (no GPU: every call is refused, at the latest for its missing workspace).

The promise: refused where some singular value in [0, 1] would leave [-2, 2] on its way, or |b s^2 + c s^4| pass 24; also where
it comes so near that 16-bit rounding could take it there."""
import math
import time

import numpy as np
import pytest

from paper_2302_07475_b200 import binding, build as B
from test_operators_host import C, FAKE, INV, WS, mat, ortho

USUAL = [(5, C), (32, C), (32, (1.5, -0.5, 0.0)), (32, (1.875, -1.25, 0.375)), (32, (2.0, -1.5, 0.5)), (1, (2.0, 0.0, 0.0)), (32, (1.02, 0.0, 0.0)),
         (1, (0.0, 0.0, 0.0)), (3, (-1.0, 0.0, 0.0))]


@pytest.fixture(scope="module")
def lib():
    B.build()
    return binding.load()


def accepted(lib, steps, coeffs):
    code = ortho(lib, steps=steps, coeffs=tuple(float(np.float32(v)) for v in coeffs), ws=None)
    assert code in (INV, WS)
    return code == WS


def extremes(steps, coeffs, points):
    """Largest |s| and |b s^2 + c s^4| on the way from these starting points (those that pass 1e3 stay there)."""
    a, b, c = (float(np.float32(v)) for v in coeffs)
    s, most, q_most = points.copy(), 0.0, 0.0
    for _ in range(steps):
        q = b * s ** 2 + c * s ** 4
        s = np.clip(s * (a + q), -1e3, 1e3)
        most, q_most = max(most, np.abs(s).max()), max(q_most, np.abs(q).max())
    return most, q_most


@pytest.mark.parametrize("steps,coeffs,start", [(15, (3.5453, -7.3801, 2.8220), 0.998475), (10, (1.8256, -4.3408, 1.4911), 0.996450)])
def test_values_that_diverge_between_the_points_of_a_grid(lib, steps, coeffs, start):
    assert extremes(steps, coeffs, np.linspace(0, 1, 1025))[0] < 1.7                    # a grid does not see them
    assert extremes(steps, coeffs, np.linspace(start - 1e-4, start + 1e-4, 2001))[0] > 100
    assert not accepted(lib, steps, coeffs)


@pytest.mark.parametrize("steps,coeffs", USUAL)
def test_usual_coefficients_are_accepted(lib, steps, coeffs):
    assert accepted(lib, steps, coeffs)


def test_whatever_leaves_the_range_is_refused_and_what_keeps_a_distance_accepted(lib):
    r = np.random.default_rng(0)
    fine, noisy = np.linspace(0, 1, 20001), np.linspace(0, 1, 2001)
    seen = [0, 0]
    for _ in range(1000):
        steps, coeffs = int(r.integers(1, 16)), (r.uniform(-1, 5), r.uniform(-10, 3), r.uniform(-1, 6))
        most, q = extremes(steps, coeffs, fine)
        if most > 2 or q > 24:
            assert not accepted(lib, steps, coeffs), (steps, coeffs)
            seen[0] += 1
        elif accepted(lib, steps, coeffs):                   # then 11-bit rounding does not take it out of fp16's range
            s, (a, b, c) = noisy.copy(), coeffs
            for _ in range(steps):
                s = s * (1 + r.uniform(-2.0 ** -11, 2.0 ** -11, s.shape))
                s = s * (a + b * s ** 2 + c * s ** 4)
                assert np.abs(s).max() < 3.9, (steps, coeffs)
            seen[1] += 1
        else:                                                # near the limit: some value next to [0, 1] leaves it
            wider = np.linspace(0, (1 + 2.0 ** -9) ** steps, 20001)
            assert extremes(steps, coeffs, wider)[0] > 1.5 or extremes(steps, coeffs, wider)[1] > 20, (steps, coeffs)
    assert min(seen) > 100


def test_large_and_small_coefficients(lib):
    big, tiny = 3.0e38, 1e-45
    for coeffs in ((big, 0, 0), (0, big, 0), (0, 0, big), (big, -big, big), (1, tiny, -big)):
        assert not accepted(lib, 2, coeffs)
    for coeffs in ((1, tiny, 0), (1, 0, tiny), (1, tiny, tiny), (1, -tiny, tiny), (tiny, tiny, tiny)):
        assert accepted(lib, 5, coeffs)
    for bad in (math.inf, -math.inf, math.nan):
        for k in range(3):
            coeffs = [1.0, 0.0, 0.0]
            coeffs[k] = bad
            assert ortho(lib, coeffs=tuple(coeffs), ws=None) == INV


def test_the_check_costs_little(lib):
    """32 steps; looking at a thousand values took 100 us and more (a whole small update takes 30)."""
    g, out, times = mat(), mat(), []
    for _ in range(200):
        t = time.perf_counter()
        lib.s3gd_orthogonalise(g, out, 1, 8, 8, 32, *C, 1e-7, -1, None, 0, None)
        times.append(time.perf_counter() - t)
    assert min(times) < 40e-6
