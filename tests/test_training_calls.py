"""What the Python entry points of the optimiser hand to the library when arguments are left out (CPU, without a launch)."""
import types

import numpy as np
import pytest

import paper_2203_00854_amd as P
from oracle import adamw as A
from paper_2203_00854_amd import binding as B


class Calls:
    """In place of the compiled module: keeps the arguments of every call."""

    def __init__(self):
        self.seen = []

    def adamw_step(self, *args):
        self.seen.append(args)
        return B.FF_OK


@pytest.fixture
def calls(monkeypatch):
    stand_in = Calls()
    monkeypatch.setattr(B, "calls", lambda: stand_in)
    return stand_in


PLAN = types.SimpleNamespace(desc=B.AdamWDesc(P.FF_F32, P.FF_F32, 8, 1), plan=None, stream=0)


def test_steps_without_a_seed_keep_the_mean(calls):
    """8-bit states over 400 steps, rounded by the oracle with the seeds that the entry point passes.  A rounding is off by at most a code's distance, v / 8,
    with a deviation of half of that; over the steps they add up as beta2's powers do, to v / 16 (1 - beta2^2)^(-1/2) at most."""
    n, steps, b1, b2 = 1 << 14, 400, 0.9, 0.99
    for step in range(1, steps + 1):
        P.ff_adamw_step(PLAN, step, lr=1e-3, betas=(b1, b2))
    seeds = [args[9] for args in calls.seen]
    assert len(set(seeds)) == steps
    rng = np.random.default_rng(0)
    m, v = (np.zeros(n, np.uint8), np.zeros(n // 256, np.uint8)), (np.zeros(n, np.uint8), np.zeros(n // 256, np.uint8))
    exact = np.zeros(n)
    for seed in seeds:
        g = rng.normal(size=n).astype(np.float32)
        m32, v32 = A.moments_f32(g, A.decode(*m, A.TOP_M), A.decode(*v, A.TOP_V), b1, b2)
        bits = A.dither(np.arange(n), seed)
        m, v = A.encode(m32, A.TOP_M, bits & 0xFFFF), A.encode(v32, A.TOP_V, bits >> 16)
        exact = b2 * exact + (1 - b2) * g.astype(np.float64) ** 2
    held = A.decode(*v, A.TOP_V).astype(np.float64)
    deviation = 1 / 16 / np.sqrt(1 - b2 ** 2) * np.sqrt((exact ** 2).mean()) / exact.mean()
    assert abs(held.mean() / exact.mean() - 1) < 6 * deviation / np.sqrt(n)


def test_a_seed_that_is_given_is_passed(calls):
    for seed in (0, 7, 1 << 31):
        P.ff_adamw_step(PLAN, 3, lr=1e-3, seed=seed)
    assert [args[9] for args in calls.seen] == [0, 7, 1 << 31]


@pytest.mark.parametrize("bits", [32, 8])
def test_states_of_tensors_that_are_given_once(bits):
    """What a module's parameters() gives can be gone through once only."""
    import torch
    params = [torch.zeros(n) for n in (300, 1, 0)]
    states, want = P.adamw_states((p for p in params), bits), P.adamw_states(params, bits)
    assert {k: [(t.numel(), t.dtype) for t in ts] for k, ts in states.items()} == {k: [(t.numel(), t.dtype) for t in ts] for k, ts in want.items()}
    assert [t.numel() for t in states["v"]] == [300, 1, 0] and all(not t.any() for ts in states.values() for t in ts)
