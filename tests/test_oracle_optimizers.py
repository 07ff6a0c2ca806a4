"""Pins of the fp64 oracle of Muon and AdamW: closed forms that the formulas have to meet."""
import numpy as np
import pytest

from oracle.optimizers_oracle import adamw_step, muon_step, newton_schulz

QUINTIC = ((3.4445, -4.7750, 2.0315),) * 5
POLAR = ((1.875, -1.25, 0.375),) * 30          # s -> (15 s - 10 s^3 + 3 s^5) / 8: fixed point 1, converges from (0, 1]


def _scalar(s, coeffs):
    for a, b, c in coeffs:
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("shape", [(1, 1), (1, 5), (6, 6), (9, 4), (4, 9)])
def test_iteration_acts_on_the_singular_values(shape):
    rng = np.random.default_rng(0)
    a = rng.standard_normal(shape)
    u, s, vt = np.linalg.svd(a, full_matrices=False)
    want = (u * _scalar(s / (np.linalg.norm(a) + 1e-7), QUINTIC)) @ vt
    assert np.allclose(newton_schulz(a, QUINTIC), want, atol=1e-12)


def test_converging_coefficients_give_the_polar_factor():
    a = np.random.default_rng(1).standard_normal((12, 7))
    u, _, vt = np.linalg.svd(a, full_matrices=False)
    assert np.allclose(newton_schulz(a, POLAR), u @ vt, atol=1e-9)


def test_zero_and_non_finite_matrices():
    assert np.all(newton_schulz(np.zeros((3, 4)), QUINTIC, eps=0.0) == 0)
    a = np.ones((3, 4))
    a[1, 2] = np.inf
    assert np.all(np.isnan(newton_schulz(a, QUINTIC)))


def test_muon_step_without_history_is_the_scaled_orthogonalised_gradient():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((5, 8)), rng.standard_normal((5, 8))
    new_x, m, _ = muon_step(x, g, np.zeros_like(g), QUINTIC, 0.9, 0.1, 0.5, 2.0)
    assert np.allclose(m, g)
    assert np.allclose(new_x, 0.95 * x - 0.2 * newton_schulz(1.9 * g, QUINTIC, 1e-7))


def test_adamw_first_step_moves_by_lr_against_the_sign():
    x, g = np.array([1.0, -2.0, 3.0]), np.array([0.5, -4.0, 1e-3])
    new_x, m, v = adamw_step(x, g, np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.999, 0.0, 0.01)
    assert np.allclose(new_x, 0.999 * x - 0.1 * np.sign(g))
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 1e-3 * g * g)
