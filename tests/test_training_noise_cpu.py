"""The numbers that 8-bit states are rounded with, where the caller gives none: taken from the step."""
import numpy as np

import paper_2512_14628_amd as pkg
from tests.ref_e4m3 import round_down_on_grid, rounding_numbers


def noise(step, given=0):
    return pkg.hsadmm_adamw_coefficients(1e-3, 0.9, 0.999, 0.0, step, given)[3]


def test_numbers_given_are_kept_and_steps_without_one_differ():
    assert noise(1, 7) == 7 and noise(5, 0xFFFFFFFF) == 0xFFFFFFFF
    numbers = [noise(t) for t in range(1, 4097)] + [noise(2 ** 40 + t) for t in range(64)]
    assert len(set(numbers)) == len(numbers)
    # of an element and two steps in a row: no correlation beyond five standard deviations (2^-8 of 65536 elements)
    u = [rounding_numbers(1 << 16, 1, noise(t))[0] - 0.5 for t in (1, 2, 3, 1000, 1001)]
    for a, b in ((0, 1), (1, 2), (0, 2), (3, 4)):
        assert abs((u[a] * u[b]).mean() * 12) < 5 * 2.0 ** -8


def test_a_second_moment_under_gradients_stays_near_its_value_without_numbers_from_the_caller():
    """Roots of a second moment held as the header says (blocks of 256, e4m3, rounded with the step's numbers), under unit
    normal gradients, against the same moment in 64 bits.

    Rounding leaves a root's mean alone, so it adds its variance to the moment's.  Between two neighbouring codes at a distance
    s, d from one of them, the variance is at most s d; s is at most r / 8.  d is at most what the root moved by and what the
    block's scale moved it by, (1 - beta) |g^2 - v| / 2r each, of mean below (1 - beta) 1.5 V / 2r (0.97 V for v = V, the rest for
    v's own spread).  A moment forgets 1 - beta of its value a step, so it settles at most at (1 + 2 * 1.5 / 16) V, and never
    below V.  The mean of 8192 elements of a spread of a half: five standard deviations are 0.03."""
    n, beta, steps = 8192, 0.99, 600
    rng = np.random.default_rng(0)
    exact, r = np.zeros(n), np.zeros(n)
    for t in range(1, steps + 1):
        g2 = rng.standard_normal(n) ** 2
        exact = beta * exact + (1 - beta) * g2
        root = np.sqrt(beta * r * r + (1 - beta) * g2).reshape(-1, 256)
        scale = root.max(1, keepdims=True) / 448
        u = rounding_numbers(n, 1, noise(t))[0].reshape(-1, 256)
        r = (np.maximum(round_down_on_grid(np.minimum(root / scale, 448), u), 2.0 ** -9) * scale).reshape(-1)
    ratio = (r * r).mean() / exact.mean()
    assert 0.97 < ratio < 1.19 + 0.03, ratio
