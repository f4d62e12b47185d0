"""GPU parity of ff_orthogonalise and ff_muon_step on tiles of 128, alone and many, in lists of ragged matrices either way round.

The reference is float64 on the GPU.  A pair of float16 is off by 1.5 times as much as a float32 value and sums are float32, so errors in norm are held to twice those of the same formulas
in float32 (the derivation is that of test_gpu_newton_schulz.py); of a result in bfloat16, and of weights, their own roundings come on top.
"""
import pytest
import torch

import paper_2203_00854_amd as P
from oracle import muon as M
from test_gpu_newton_schulz import DEV, DTYPES, gradients, newton_schulz

pytestmark = pytest.mark.gpu
HALF = {torch.float32: M.U, torch.bfloat16: 2.0 ** -8}


# A of (1810, 1900) has 120 tiles of 128, X 225; A of (2570, 2600) 231, X 441.  45 matrices of (300, 700) have 270 and 810.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", [(1, 1810, 1900), (1, 1900, 1810), (1, 2570, 2600), (1, 2600, 2570), (45, 300, 700), (45, 700, 300)])
def test_orthogonalise(count, rows, cols, dtype):
    x = torch.stack([gradients(rows, cols, i) for i in range(count)]).to(DTYPES[dtype])
    out = P.ff_orthogonalise(x)
    for i in sorted({0, count // 2, count - 1}):
        want = newton_schulz(x[i], torch.float64)
        plain = (newton_schulz(x[i], torch.float32).double() - want).norm()
        off = (out[i].double() - want).norm()
        print(f"{rows} x {cols} {dtype}: {off / want.norm():.2e}, float32 {plain / want.norm():.2e}", flush=True)
        assert off <= 2 * plain + (0.0 if dtype == "f32" else HALF[x.dtype] * want.norm())
    assert torch.equal(P.ff_orthogonalise(x, out=x), out)


MANY = [(300, 700), (700, 300), (130, 1000), (1000, 130), (450, 450)] * 11         # 11 (6 + 6 + 3 + 3 + 10) = 308 tiles of A, more of X: many of 128
SMALL = [(20, 30), (128, 128), (5, 100), (64, 64), (1, 7)]
LISTS = {"some": [(1810, 1900), (300, 150), (20, 30)],                              # 120 + 3 + 1 tiles of A: of 64; 225 + 6 + 1 of X: some of 128
         "some_tall": [(2600, 2570), (33, 200)],                                    # 231 + 1 of A: some of 128; many of X
         "many_with_small_among_them": MANY + SMALL,
         "many_with_small_behind_them": MANY + SMALL * 20}


@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("master", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("name", LISTS)
def test_steps(name, param, grad):
    shapes = LISTS[name]
    kind = torch.float32 if param == "f32" else torch.bfloat16
    each = [gradients(*s, i) for i, s in enumerate(shapes)]
    g = [0.01 * t for t in each] if grad == "f32" else [(0.01 * t).to(torch.bfloat16) for t in each]
    m = [0.005 * gradients(*s, 1000 + i) for i, s in enumerate(shapes)]
    p = [gradients(*s, 2000 + i).to(kind) for i, s in enumerate(shapes)]
    master = [t.float() for t in p] if param == "master" else None
    was = [[t.clone() for t in (master or p)], [t.clone() for t in m]]
    lr, beta, decay = 0.02, 0.95, 0.125
    P.ff_muon_step(P.make_muon_plan(p, g, m, master=master, weight_decay=decay), lr, beta=beta)
    for i, s in enumerate(shapes):
        g64, m64, w64 = g[i].double(), was[1][i].double(), was[0][i].double()
        m64, now = beta * m64 + (1 - beta) * g64, (1 - beta) * g64
        # 1 - beta, beta, two products, a sum: of terms of any sign
        assert bool(((m[i].double() - m64).abs() <= 6 * M.U * (beta * was[1][i].double().abs() + now.abs())).all()), s
        exact = newton_schulz(beta * m64 + now, torch.float64)
        m32 = beta * was[1][i] + (1 - beta) * g[i].float()
        plain = (newton_schulz(beta * m32 + (1 - beta) * g[i].float(), torch.float32).double() - exact).norm()
        size = lr * M.step_size("spectral", *s)
        want = w64 - lr * decay * w64 - size * exact
        after = (master or p)[i].double()
        # lr, the decay, the size, three products and two sums
        bound = 2 * size * plain + 8 * M.U * (w64.abs() + size * exact.abs()).norm()
        if master:
            assert torch.equal(p[i], master[i].to(torch.bfloat16)), s
        else:
            bound = bound + HALF[kind] * want.norm()
        assert (after - want).norm() <= bound, (s, (after - want).norm(), bound)


@pytest.mark.parametrize("rows,cols", [(32768, 32768), (32768, 1), (1, 32768), (130, 32768), (32768, 130)])
def test_largest_matrices(rows, cols):
    """One step of the largest sides, whose X and A reach 4 GiB each: some rows of it in float64, from X alone."""
    g = gradients(rows, cols, rows + cols)                # (large singular values, or the products would be small beside a X)
    some = sorted({0, 1, rows // 3, rows - 2, rows - 1} & set(range(rows)))
    out = P.ff_orthogonalise(g, steps=1)
    a, b, c = M.COEFFICIENTS

    def product(left, turned):                              # by parts of the rows of g, in float64
        parts = [g[at:at + 4096].double() for at in range(0, rows, 4096)]
        if turned:
            return torch.cat([left @ p.mT.contiguous() for p in parts], 1)
        return sum(left[:, 4096 * i:4096 * i + p.shape[0]] @ p for i, p in enumerate(parts))

    length = sum(g[at:at + 4096].double().square().sum() for at in range(0, rows, 4096)).sqrt() + 1e-7
    x = g[some].double() / length
    once = product(product(x, True), False) / length ** 2             # X X^T X
    want = a * x + b * once + c * product(product(once, True), False) / length ** 2
    off = (out[some].double() - want).norm() / want.norm()
    # a value of X, A, B: 2^-23 at most, in a sum of terms of any sign no more of it in norm; float32 sums of n terms of one sign (A's diagonal) or any: 8 deviations of 2^-24 (n / 2)^(1/2)
    bound = (4 * 2 + 8 * (max(rows, cols) / 2) ** 0.5) * M.U * (a - b + c) * x.norm() / want.norm()
    print(f"{rows} x {cols}: {off:.2e} of {bound:.2e}", flush=True)
    assert off <= bound
