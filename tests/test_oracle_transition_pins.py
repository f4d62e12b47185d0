"""Pins of the transition's and the Muon step's oracles: differences, closed forms, the mathematics of the polynomial (CPU)."""
import numpy as np
import pytest

from oracle import muon as M
from oracle import transition as T


def problem(rows=5, c=4, f=6, seed=0):
    rng = np.random.default_rng(seed)
    return [rng.normal(size=s) for s in ((rows, c), (f, c), (f, c), (c, f), (rows, c))]


@pytest.mark.parametrize("kind", ["silu", "gelu", "sigmoid"])
def test_slopes_are_the_activations_differences(kind):
    a = np.linspace(-9, 9, 301)
    near = (T.act(kind, a + 1e-5) - T.act(kind, a - 1e-5)) / 2e-5
    assert np.abs(near - T.slope(kind, a)).max() < 1e-9
    assert np.abs(T.slope(kind, a)).max() <= T.STEEPEST[kind]
    assert np.abs(np.diff(T.slope(kind, a)) / np.diff(a)).max() <= T.BEND[kind]


def test_values_by_hand():
    x, w = np.array([[1.0, 2.0]]), np.eye(2)
    s = 1 / (1 + np.exp(-np.array([1.0, 2.0])))
    assert np.allclose(T.forward(x, w, 3 * w, w, "silu"), 3 * np.array([1.0, 4.0]) * s, rtol=1e-14)
    assert np.allclose(T.forward(x, w, 3 * w, w, "sigmoid", residual=x), x + 3 * np.array([1.0, 2.0]) * s, rtol=1e-14)
    assert np.allclose(T.act("gelu", np.array([1.0])), 0.8413447460685429, rtol=1e-14)


@pytest.mark.parametrize("kind", ["silu", "gelu", "sigmoid"])
def test_gradients_are_differences(kind):
    x, w_a, w_b, w_o, dy = problem()
    mask = np.array([1, 0, 1, 1, 0.0])
    grads = T.backward(x, w_a, w_b, w_o, dy, kind, mask)
    args = [x, w_a, w_b, w_o]
    loss = lambda: (T.forward(*args, kind, mask) * dy * mask[:, None]).sum()  # noqa: E731
    for t, g in zip(args, grads):
        for i in np.ndindex(*t.shape):
            keep = t[i]
            t[i] = keep + 1e-5
            up = loss()
            t[i] = keep - 1e-5
            down = loss()
            t[i] = keep
            assert abs((up - down) / 2e-5 - g[i]) < 1e-8 * (1 + abs(g[i]))


def test_masked_rows_reach_nothing():
    x, w_a, w_b, w_o, dy = problem()
    mask = np.array([1, 0, 1, 1, 0.0])
    want = T.forward(x, w_a, w_b, w_o, "silu", mask), T.backward(x, w_a, w_b, w_o, dy, "silu", mask)
    x[1], dy[4], x[4] = np.nan, np.inf, -np.inf
    assert np.array_equal(T.forward(x, w_a, w_b, w_o, "silu", mask), want[0]) and not want[0][[1, 4]].any()
    for a, b in zip(T.backward(x, w_a, w_b, w_o, dy, "silu", mask), want[1]):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("half", [T.U, 2.0 ** -8])
@pytest.mark.parametrize("kind", ["silu", "gelu", "sigmoid"])
def test_bounds_hold_for_rounded_evaluations(kind, half):
    """The formulas in float32, rounded as the kernels round, stay within the bounds; bounds stay well below the values."""
    import torch
    x, w_a, w_b, w_o, dy = problem(40, 24, 32, 3)
    keep = torch.float32 if half == T.U else torch.bfloat16
    r = lambda t: torch.tensor(np.asarray(t, np.float32)).to(keep).float().numpy()  # noqa: E731
    x, w_a, w_b, w_o, dy = (r(t) for t in (x, w_a, w_b, w_o, dy))
    a, b = x @ w_a.T, x @ w_b.T
    h, dh = r(T.act(kind, a) * b), dy @ w_o
    da, db = r(dh * b * T.slope(kind, a)), r(dh * T.act(kind, a))
    got = [r(h @ w_o.T), r(da @ w_a + db @ w_b), r(da.T @ x), r(db.T @ x), r(dy.T @ h)]
    wide = [t.astype(np.float64) for t in (x, w_a, w_b, w_o, dy)]
    want = [T.forward(*wide[:4], kind), *T.backward(*wide, kind)]
    bound = [T.forward_bound(*wide[:4], kind, half), *T.backward_bound(*wide, kind, half, half)]
    for g, w, e in zip(got, want, bound):
        assert np.all(np.abs(g - w) <= e)
        # (sums of up to 40 terms, three products in a row, each (n + 2) units of sums of magnitudes some five times the sums: thousands of units)
        assert np.median(e) < (1e-3 if half == T.U else 0.5) * np.median(np.abs(w))


@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (7, 3), (6, 6)])
def test_orthogonalise_acts_on_singular_values(shape):
    """U diag(s) V^T becomes U diag(p(...p(s))) V^T."""
    g = np.random.default_rng(1).normal(size=shape)
    u, s, v = np.linalg.svd(g, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-7)
    a, b, c = M.COEFFICIENTS
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(M.orthogonalise(g), u * s @ v, atol=1e-12)
    assert np.all(np.abs(s) < 1.3)


def test_cubic_polynomial_converges_to_the_polar_factor():
    g = np.random.default_rng(2).normal(size=(4, 9))
    u, _, v = np.linalg.svd(g, full_matrices=False)
    assert np.allclose(M.orthogonalise(g, steps=40, coefficients=(1.5, -0.5, 0.0), eps=0.0), u @ v, atol=1e-12)


def test_roundings_are_of_the_size_of_float32():
    g = np.random.default_rng(3).normal(size=(24, 40))
    low = np.asarray(g, np.float32)
    x = low / np.float32(np.linalg.norm(low) + 1e-7)
    a, b, c = (np.float32(q) for q in M.COEFFICIENTS)
    for _ in range(5):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    total, most = M.roundings(low)
    off = x - M.orthogonalise(low)
    assert np.linalg.norm(off) < total < 1e-3 * np.linalg.norm(x) and np.abs(off).max() < most


def test_muon_step_by_hand():
    """1 x 1: the update is p(...p(sign)) of any size."""
    w, m = M.step(np.array([[2.0]]), np.array([[-3.0]]), np.array([[1.0]]), lr=0.1, beta=0.5, decay=0.25, nesterov=False, eps=0.0)
    s = 1.0
    for _ in range(5):
        s = sum(q * s ** e for q, e in zip(M.COEFFICIENTS, (1, 3, 5)))
    assert m[0, 0] == -1.0 and np.isclose(w[0, 0], 2.0 - 0.1 * (0.5 - s))
    assert M.step_size("spectral", 8, 2) == 2 and M.step_size("spectral", 2, 8) == 1 and M.step_size("rms", 4, 25) == 1
