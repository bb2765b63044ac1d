"""The oracles of the Muon step and the router, pinned by closed forms, singular values and differences (CPU)."""
import numpy as np
import pytest

from oracle import muon_oracle as M
from oracle import router_oracle as R

ABC = (3.4445, -4.7750, 2.0315)


def _scalar(x, coefficients, steps):
    for a, b, c in np.broadcast_to(np.asarray(coefficients, dtype=np.float32).astype(np.float64), (steps, 3)):
        x = a * x + b * x ** 3 + c * x ** 5
    return x


@pytest.mark.parametrize("m,n", [(1, 1), (1, 9), (7, 3), (12, 12), (5, 40)])
def test_orthogonalize_moves_singular_values(m, n):
    g = np.random.default_rng(m * 100 + n).standard_normal((m, n))
    u, s, v = np.linalg.svd(g / (np.linalg.norm(g) + 1e-7), full_matrices=False)
    want = (u * _scalar(s, ABC, 5)) @ v
    np.testing.assert_allclose(M.orthogonalize(g, ABC, 5, 1e-7), want, rtol=0, atol=1e-10)


def test_steps_may_have_coefficients_of_their_own():
    g = np.random.default_rng(0).standard_normal((6, 11))
    per = np.array([[3.0, -3.2, 1.2], [2.0, -1.5, 0.5], [1.875, -1.25, 0.375]])
    u, s, v = np.linalg.svd(g / np.linalg.norm(g), full_matrices=False)
    np.testing.assert_allclose(M.orthogonalize(g, per, 3, 0.0), (u * _scalar(s, per, 3)) @ v, rtol=0, atol=1e-10)


@pytest.mark.parametrize("m,n", [(1, 5), (16, 16), (64, 200), (130, 70)])
def test_rounded_form_is_near(m, n):
    """2^-9, what the header says of the kernels' operands."""
    g = np.random.default_rng(m + n).standard_normal((m, n))
    want = M.orthogonalize(g, ABC, 5, 1e-7)
    got = M.orthogonalize_rounded(g, ABC, 5, 1e-7)
    assert np.linalg.norm(got - want) <= 2.0 ** -9 * np.linalg.norm(want)


@pytest.mark.parametrize("m,n", [(16, 60), (200, 64), (130, 400)])
def test_rounded_form_of_two_steps_taken_as_one_is_near(m, n):
    g = np.random.default_rng(m + n).standard_normal((m, n))
    for steps in (2, 5):
        want = M.orthogonalize(g, ABC, steps, 1e-7)
        assert np.linalg.norm(M.orthogonalize_rounded(g, ABC, steps, 1e-7, True) - want) <= 2.0 ** -9 * np.linalg.norm(want)


def test_muon_step_of_a_single_value():
    p, m = M.muon_step([[2.0]], [[-0.5]], [[0.0]], ABC, 5, 0.0, 0.1, 0.9, True, 0.01)
    np.testing.assert_allclose(m, [[-0.05]])
    np.testing.assert_allclose(p, [[2.0 * (1 - 0.001) + 0.1 * _scalar(1.0, ABC, 5)]])


def test_uniform_router_has_balance_one():
    f = R.forward(np.zeros((12, 4)), 4)
    np.testing.assert_allclose(f["losses"], [1.0, np.log(4.0) ** 2])
    assert (f["indices"] == np.arange(4)).all() and (f["counts"] == [12, 12, 12, 12, 12]).all()


def test_router_masks_and_ties():
    x = np.array([[1.0, 3.0, 3.0, -np.inf], [-np.inf] * 4, [0.0, -np.inf, -np.inf, -np.inf], [5.0, 5.0, 5.0, 5.0]])
    f = R.forward(x, 2, taken=np.array([True, True, True, False]))
    assert (f["indices"] == [[1, 2], [-1, -1], [0, -1], [-1, -1]]).all()
    assert (f["counts"] == [1, 1, 1, 0, 2]).all()
    np.testing.assert_allclose(f["weights"], [[0.5, 0.5], [0, 0], [1, 0], [0, 0]])


@pytest.mark.parametrize("renormalize", [True, False])
def test_router_gradient_is_that_of_differences(renormalize):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 7))
    x[1, 2] = x[1, 4] = -np.inf
    f = R.forward(x, 3, taken=np.array([True, True, False, True, True]))
    dw, dl = rng.standard_normal((5, 3)), np.array([0.7, -0.3])
    got = R.backward(x, f["indices"], f["counts"], dw, dl, renormalize)
    assert (got[2] == 0).all() and (got[1, [2, 4]] == 0).all()
    h = 1e-6
    for i in range(5):
        for e in range(7):
            if np.isneginf(x[i, e]):
                continue
            up, down = x.copy(), x.copy()
            up[i, e] += h
            down[i, e] -= h
            want = (R.total(up, f["indices"], f["counts"], dw, dl, renormalize) - R.total(down, f["indices"], f["counts"], dw, dl, renormalize)) / (2 * h)
            assert abs(got[i, e] - want) < 1e-8
