"""Float64 oracle of the gated transition (ff_gated_transition_forward, ff_gated_transition_backward), with bounds of what roundings can add up to.

    a = x Wa^T;  b = x Wb^T;  h = act(a) b;  y = h Wo^T
    dh = dy Wo;  da = dh b act'(a);  db = dh act(a);  dx = da Wa + db Wb;  dWa = da^T x;  dWb = db^T x;  dWo = dy^T h

Rows whose mask is 0 take no part, whatever they hold.
"""
import numpy as np
from scipy.special import erf, erfc, expit

U = 2.0 ** -24                     # half a step of float32, relative to the value


def act(kind, a):
    if kind == "silu":
        return a * expit(a)
    if kind == "gelu":
        return a * 0.5 * erfc(-a / np.sqrt(2))
    return expit(a)


def slope(kind, a):
    s = expit(a)
    if kind == "silu":
        return s * (1 + a * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + erf(a / np.sqrt(2))) + a * np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    return s * (1 - s)


STEEPEST = {"silu": 1.1, "gelu": 1.13, "sigmoid": 0.25}       # of act
BEND = {"silu": 0.5, "gelu": 0.8, "sigmoid": 0.1}             # of act'


def live(t, mask):
    t = np.asarray(t, np.float64)
    return t if mask is None else np.where(np.asarray(mask)[:, None] != 0, t, 0.0)


def forward(x, w_a, w_b, w_o, kind, mask=None, residual=None):
    x = live(x, mask)
    y = (act(kind, x @ w_a.T) * (x @ w_b.T)) @ w_o.T
    return y if residual is None else y + residual


def backward(x, w_a, w_b, w_o, dy, kind, mask=None):
    x, dy = live(x, mask), live(dy, mask)
    a, b = x @ w_a.T, x @ w_b.T
    gate, dh = act(kind, a), dy @ w_o
    da, db = dh * b * slope(kind, a), dh * gate
    return da @ w_a + db @ w_b, da.T @ x, db.T @ x, dy.T @ (gate * b)


# ---- bounds: a sum of n products in float32 is off by at most (n + 2) U times the sum of their magnitudes (two roundings a term leave room for any order), and
# an operand's error e adds e times the other operand's magnitude.  half: what rounding a tensor to its type adds, relative; the activation's own error is 16 + |a| units.
def _product(p, ep, q, eq):
    """Bound of the error of p @ q.T."""
    n = p.shape[1]
    return 2 * (n + 2) * U * (np.abs(p) @ np.abs(q).T) + ep @ (np.abs(q) + eq).T + np.abs(p) @ eq.T


def _hidden(x, w_a, w_b, kind, half):
    zx, zw = np.zeros_like(x), np.zeros_like(w_a)
    a, b = x @ w_a.T, x @ w_b.T
    ea, eb = _product(x, zx, w_a, zw), _product(x, zx, w_b, zw)
    gate = act(kind, a)
    eg = STEEPEST[kind] * ea + (16 + np.abs(a)) * U * (np.abs(gate) + STEEPEST[kind] * ea) + 1e-37
    h = gate * b
    eh = eg * (np.abs(b) + eb) + np.abs(gate) * eb
    eh = eh + (half + 2 * U) * (np.abs(h) + eh)
    return a, b, ea, eb, gate, eg, h, eh


def forward_bound(x, w_a, w_b, w_o, kind, half, mask=None, residual=None):
    x = live(x, mask)
    *_, h, eh = _hidden(x, w_a, w_b, kind, half)
    y = h @ w_o.T
    e = _product(h, eh, w_o, np.zeros_like(w_o))
    if residual is not None:
        y = y + residual
    return e + (half + 2 * U) * (np.abs(y) + e) + 1e-37


def backward_bound(x, w_a, w_b, w_o, dy, kind, half, half_w, mask=None):
    """half_w: the rounding of the weights' gradients."""
    x, dy = live(x, mask), live(dy, mask)
    a, b, ea, eb, gate, eg, h, eh = _hidden(x, w_a, w_b, kind, half)
    dh, zero = dy @ w_o, np.zeros_like
    edh = _product(dy, zero(dy), w_o.T, zero(w_o.T))
    s = slope(kind, a)
    es = BEND[kind] * ea + (32 + 2 * np.abs(a)) * U * (np.abs(s) + 1)
    da, db = dh * b * s, dh * gate
    eda = edh * (np.abs(b) + eb) * (np.abs(s) + es) + np.abs(dh) * (eb * (np.abs(s) + es) + np.abs(b) * es)
    edb = edh * (np.abs(gate) + eg) + np.abs(dh) * eg
    eda, edb = (e + (half + 4 * U) * (np.abs(t) + e) for t, e in ((da, eda), (db, edb)))
    rounded = lambda t, e, by: e + (by + 2 * U) * (np.abs(t) + e) + 1e-37  # noqa: E731
    dx = da @ w_a + db @ w_b
    edx = _product(np.concatenate([da, db], 1), np.concatenate([eda, edb], 1), np.concatenate([w_a, w_b]).T, np.zeros((dx.shape[1], 2 * a.shape[1])))
    out = [rounded(dx, edx, half)]
    for p, ep, q, eq in ((da, eda, x, zero(x)), (db, edb, x, zero(x)), (dy, zero(dy), h, eh)):
        out.append(rounded(p.T @ q, _product(p.T, ep.T, q.T, eq.T), half_w))
    return out
