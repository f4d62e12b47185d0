"""Pins of the training oracles (oracle/layernorm_train.py, oracle/adamw.py): gradients against central differences and
torch's float64 autograd, the step against torch's AdamW in float64, the 8-bit codes against what they promise.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import adamw as A
from oracle import layernorm_train as L


@pytest.mark.parametrize("rows,c", [(1, 1), (3, 2), (5, 7), (4, 32)])
def test_layernorm_gradients(rows, c):
    rng = np.random.default_rng(rows * 100 + c)
    s, dy, dsum = (rng.normal(size=(rows, c)) for _ in range(3))
    gamma, beta = rng.normal(size=c), rng.normal(size=c)
    eps = 1e-3
    dx, dgamma, dbeta = L.backward(s, gamma, dy, eps, dsum)
    ts, tg, tb = (torch.tensor(a, requires_grad=True) for a in (s, gamma, beta))
    y = torch.nn.functional.layer_norm(ts, (c,), tg, tb, eps)
    assert np.max(np.abs(y.detach().numpy() - L.forward(s, gamma, beta, eps)[0])) < 1e-11
    ((y * torch.tensor(dy)).sum() + (ts * torch.tensor(dsum)).sum()).backward()
    for got, want in ((dx, ts), (dgamma, tg), (dbeta, tb)):
        assert np.max(np.abs(got - want.grad.numpy())) < 1e-9
    # central differences of the oracle's own forward; the step's error is of order step^2 times the third derivative
    loss = lambda s_, g_, b_: float((L.forward(s_, g_, b_, eps)[0] * dy).sum() + (s_ * dsum).sum())  # noqa: E731
    for at, arg, grad in ((0, s, dx), (1, gamma, dgamma), (2, beta, dbeta)):
        for i in rng.integers(0, arg.size, 4):
            lo, hi = [s, gamma, beta], [s, gamma, beta]
            lo[at], hi[at] = arg.copy(), arg.copy()
            lo[at].flat[i] -= 1e-6
            hi[at].flat[i] += 1e-6
            assert abs((loss(*hi) - loss(*lo)) / 2e-6 - grad.flat[i]) < 1e-4 * max(1.0, abs(grad.flat[i]))


def test_step_against_torch():
    rng = np.random.default_rng(5)
    w = torch.tensor(rng.normal(size=50), requires_grad=True)
    opt = torch.optim.AdamW([w], lr=3e-3, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.05)
    mine, m, v = w.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.normal(size=50)
        norm = float(np.linalg.norm(g))
        w.grad = torch.tensor(g)
        torch.nn.utils.clip_grad_norm_([w], 2.0)
        opt.step()
        mine, m, v = A.step(mine, g, m, v, 3e-3, 0.9, 0.99, 1e-7, 0.05, t, A.clip_factor(norm, 2.0))
        assert np.max(np.abs(mine - w.detach().numpy())) < 1e-12


def test_float32_moments_are_the_formula():
    rng = np.random.default_rng(6)
    g, m, v = rng.normal(size=1000).astype(np.float32), rng.normal(size=1000).astype(np.float32), rng.random(1000).astype(np.float32)
    m32, v32 = A.moments_f32(g, m, v, 0.9, 0.999, 0.37)
    _, m64, v64 = A.step(np.zeros(1000), g, m, v, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0.37)
    u = 2.0 ** -24
    assert np.all(np.abs(m32 - m64) <= 8 * u * (np.abs(m) + np.abs(g)))
    assert np.all(np.abs(v32 - v64) <= 12 * u * v64)


VALUES = {
    "normal": lambda rng, n: rng.normal(size=n) * 1e-3,
    "wide": lambda rng, n: rng.normal(size=n) * 10.0 ** rng.uniform(-12, 2, n),
    "tiny": lambda rng, n: rng.normal(size=n) * 1e-39,
    "huge": lambda rng, n: rng.normal(size=n) * 1e37,
    "zeros": lambda rng, n: np.where(rng.random(n) < 0.9, 0.0, 1.0),
}


@pytest.mark.parametrize("kind", sorted(VALUES))
@pytest.mark.parametrize("n", [1, 255, 256, 257, 1000])
@pytest.mark.parametrize("top", [A.TOP_M, A.TOP_V])
def test_codes_hold_a_neighbour(kind, n, top):
    rng = np.random.default_rng(n)
    x = VALUES[kind](rng, n).astype(np.float32)
    x = np.abs(x) if top == A.TOP_V else x
    code, exp = A.encode(x, top, rng.integers(0, 1 << 16, n))
    held = A.decode(code, exp, top)
    assert np.all(np.isfinite(held))
    # less than one distance of codes away (with the dither's own resolution and the rounding of subnormals); a positive v may be lifted to the least code
    gap = A.spacing(x, exp, top)
    lowest = np.ldexp(1.0, np.repeat(exp.astype(np.int64), A.GROUP)[:n] - top - 126 - 3)
    assert np.all(np.abs(held.astype(np.float64) - x) <= gap * (1 + 2.0 ** -15) + 2.0 ** -149)
    assert np.all(held[x == 0] == 0)
    if top == A.TOP_V:
        fits = lowest >= 2.0 ** -149
        assert np.all(held[(x > 0) & fits] > 0)
    # codes of codes' values are themselves, whatever the dither
    again, exp2 = A.encode(held, top, rng.integers(0, 1 << 16, n))
    if np.array_equal(exp, exp2) and kind != "tiny":
        assert np.array_equal(A.decode(again, exp2, top), held)


def test_rounding_keeps_the_mean():
    rng = np.random.default_rng(8)
    n = 256 * 400
    x = (rng.normal(size=n) * 1e-2).astype(np.float32)
    for t in (1, 2, 3):
        bits = A.dither(np.arange(n), t)
        for top, b, val in ((A.TOP_M, bits & 0xFFFF, x), (A.TOP_V, bits >> 16, x * x)):
            code, exp = A.encode(val, top, b)
            off = (A.decode(code, exp, top).astype(np.float64) - val) / A.spacing(val, exp, top)
            # each of n differences has mean 0 and a deviation of at most 1/2: six deviations of their mean
            assert abs(off.mean()) < 6 * 0.5 / np.sqrt(n), (t, top, off.mean())


def test_dither_bits_are_even_and_unrelated():
    n = 1 << 16
    a, b = A.dither(np.arange(n), 7), A.dither(np.arange(n), 8)
    lo, hi = a & 0xFFFF, a >> 16
    for x in (lo, hi, b & 0xFFFF, b >> 16):
        counts = np.bincount(x >> 8, minlength=256)
        # chi-square of 255 degrees of freedom: mean 255, deviation 22.6
        assert abs(((counts - n / 256) ** 2 / (n / 256)).sum() - 255) < 6 * 22.6
    for x, y in ((lo, hi), (lo, b & 0xFFFF), (hi, b >> 16), (lo[1:], lo[:-1]), (hi[1:], hi[:-1])):
        assert abs(np.corrcoef(x, y)[0, 1]) < 6 / np.sqrt(n)


def test_groups_that_are_not_finite_hold_nan():
    x = np.ones(600, np.float32)
    x[300] = np.inf
    code, exp = A.encode(x, A.TOP_M, np.zeros(600, np.uint16))
    held = A.decode(code, exp, A.TOP_M)
    assert np.isnan(held[256:512]).all() and (held[:256] == 1).all() and (held[512:] == 1).all()
