"""Float64 oracle of the Newton-Schulz products and of the Muon step (ff_orthogonalise, ff_muon_step).

    X = G / (|G| + eps);  A = X X^T;  X = a X + (b A + c A^2) X
    m = beta m + (1 - beta) k g;  u = m or beta m + (1 - beta) k g;  w = w - lr (decay w + s O(u))

`noise` (a generator) puts into every operation what float32 sums and values of 23 bits, held as pairs of float16, would: `roundings` of the result then tells how far off an
implementation with such roundings may be, however the polynomial spreads them.
"""
import numpy as np

U = 2.0 ** -24
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _product(p, q, noise):
    z = p @ q
    if noise is None:
        return z
    # roundings of n partial sums: as those of terms of any sign, and of terms of one sign
    size = np.sqrt(p.shape[1]) * (np.abs(z) + np.sqrt((p * p) @ (q * q)))
    return z + U * size * noise.normal(size=z.shape)


def _held(z, noise):
    """As a pair of float16 values of 256 times z (or more: X): off by up to 2^-23 of z, 2^-24 or less in the mean, or by half their smallest step, 2^-33."""
    return z if noise is None else z + (U * np.abs(z) + 2.0 ** -33) * noise.normal(size=z.shape)


def orthogonalise(g, steps=5, coefficients=COEFFICIENTS, eps=1e-7, noise=None):
    g = np.asarray(g, np.float64)
    tall = g.shape[0] > g.shape[1]
    x = g.T if tall else g
    a, b, c = coefficients
    x = _held(x / (np.sqrt((x * x).sum()) + eps), noise)
    for _ in range(steps):
        gram = _held(_product(x, x.T, noise), noise)
        gram = (gram + gram.T) / 2
        poly = _held(b * gram + c * _product(gram, gram, noise), noise)
        poly = (poly + poly.T) / 2
        x = _held(a * x + _product(poly, x, noise), noise)
    return x.T if tall else x


def roundings(g, steps=5, coefficients=COEFFICIENTS, eps=1e-7, seeds=4):
    """(root of the sum of squares, largest) of what an element of orthogonalise(g) may be off: eight times the deviation of the noisy ones."""
    exact = orthogonalise(g, steps, coefficients, eps)
    off = [orthogonalise(g, steps, coefficients, eps, np.random.default_rng(s)) - exact for s in range(seeds)]
    return 8 * max(np.linalg.norm(o) for o in off), 8 * max(np.abs(o).max() for o in off)


def momentum(g, m, beta, nesterov, k=1.0):
    now = (1 - beta) * k * np.asarray(g, np.float64)
    m = beta * np.asarray(m, np.float64) + now
    return m, (beta * m + now if nesterov else m)


def step_size(kind, rows, cols):
    return np.sqrt(max(1.0, rows / cols)) if kind == "spectral" else 0.2 * np.sqrt(max(rows, cols))


def step(w, g, m, lr, beta, decay, nesterov=True, scale="spectral", steps=5, coefficients=COEFFICIENTS, eps=1e-7, k=1.0):
    """(w, m) after one step."""
    m, u = momentum(g, m, beta, nesterov, k)
    w = np.asarray(w, np.float64)
    return w - lr * (decay * w + step_size(scale, *w.shape) * orthogonalise(u, steps, coefficients, eps)), m


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))
