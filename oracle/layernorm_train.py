"""Float64 oracle of layer norm in training: forward pass with statistics, and its gradients.

Per row of c channels (FastFold Section 5.2 names the kernel; the formula is the usual one, biased variance, eps
inside the root):

    mean = sum(s) / c      rstd = (sum((s - mean)^2) / c + eps)^(-1/2)      y = (s - mean) rstd gamma + beta

and with u = (s - mean) rstd, h = dy gamma:

    dx = rstd (h - mean(h) - u mean(h u))      dgamma = sum_rows dy u      dbeta = sum_rows dy
"""
from __future__ import annotations

import numpy as np


def forward(s, gamma, beta, eps):
    """(y, mean, rstd) of s [rows, c]."""
    s = np.asarray(s, np.float64)
    mean = s.mean(1)
    rstd = (((s - mean[:, None]) ** 2).mean(1) + eps) ** -0.5
    return (s - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def backward(s, gamma, dy, eps, dsum=None):
    """(dx, dgamma, dbeta); dsum is added to dx."""
    s, dy = np.asarray(s, np.float64), np.asarray(dy, np.float64)
    mean = s.mean(1, keepdims=True)
    rstd = (((s - mean) ** 2).mean(1, keepdims=True) + eps) ** -0.5
    u = (s - mean) * rstd
    h = dy * gamma
    dx = rstd * (h - h.mean(1, keepdims=True) - u * (h * u).mean(1, keepdims=True))
    return (dx if dsum is None else dx + dsum), (dy * u).sum(0), dy.sum(0)
