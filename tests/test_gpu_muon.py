"""GPU parity of ff_orthogonalise and ff_muon_step.

The tolerance of an orthogonalised matrix is what the float64 oracle shows roundings of float32 sums and values of 23 bits grow to (oracle/muon.py: eight deviations of evaluations
with random roundings), plus the rounding of the result; momentum counts its four operations.
"""
import numpy as np
import pytest
import torch

import paper_2203_00854_amd as P
from oracle import muon as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: M.U, torch.bfloat16: 2.0 ** -8}
n64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731


def matrices(count, rows, cols, dtype, seed=0, size=1.0):
    """Few large singular values above noise, as gradients have."""
    gen = torch.Generator(DEV).manual_seed(seed)
    k = min(4, rows, cols)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    x = torch.matmul(randn(count, rows, k), randn(count, k, cols).contiguous()) + 0.3 * randn(count, rows, cols)
    return (size * x).to(DTYPES[dtype])


def check(got, g, half, **kw):
    want = M.orthogonalise(g, **kw)
    total, most = M.roundings(g, **kw)
    off = np.abs(got - want)
    assert np.linalg.norm(off) <= total + half * np.linalg.norm(want) and np.all(off <= most + half * (np.abs(want) + most)), (np.linalg.norm(off), total, off.max(), most)


SHAPES = [(1, 1, 1), (3, 1, 9), (2, 9, 1), (2, 16, 16), (3, 17, 40), (3, 40, 17), (1, 128, 64), (2, 129, 130), (1, 300, 140), (1, 140, 300), (5, 64, 8), (9, 65, 100), (2, 128, 128), (17, 150, 33), (1, 2048, 96), (1, 200, 2000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", SHAPES)
def test_orthogonalise(count, rows, cols, dtype):
    x = matrices(count, rows, cols, dtype)
    out = P.ff_orthogonalise(x)
    for i in range(count):
        check(n64(out[i]), n64(x[i]), HALF[x.dtype])
    assert torch.equal(P.ff_orthogonalise(x, out=x), out)


@pytest.mark.parametrize("kw", [dict(steps=1), dict(steps=2), dict(steps=12, coefficients=(1.5, -0.5, 0.0)), dict(eps=1.0), dict(eps=0.0)])
def test_arguments(kw):
    for rows, cols in ((48, 33), (33, 48)):
        x = matrices(1, rows, cols, "f32")[0]
        check(n64(P.ff_orthogonalise(x, **kw)), n64(x), M.U, **kw)


def test_numbers_of_steps_that_are_none():
    x = matrices(1, 24, 50, "f32")[0]
    model = Model([(3, 4)], "f32", "f32")
    before = model.all()
    for steps in (0, -1, 65, 5 - 2 ** 32, 5 + 2 ** 32):
        with pytest.raises(P.FFError):
            P.ff_orthogonalise(x, steps=steps)
        with pytest.raises(P.FFError):
            P.ff_muon_step(model.plan, 0.02, steps=steps)
    assert all(torch.equal(a, b) for a, b in zip(before, model.all()))


def test_sizes_of_values():
    """The result does not depend on how large a matrix is, down to eps and up to the type's ends."""
    x = matrices(1, 24, 50, "f32")[0]
    for size in (2.0 ** 110, 2.0 ** 30, 2.0 ** -30, 2.0 ** -110):
        check(n64(P.ff_orthogonalise(x * size, eps=0.0)), n64(x), M.U, eps=0.0)
    assert not P.ff_orthogonalise(torch.zeros(3, 20, 10, device=DEV)).any()


def test_one_bad_matrix_leaves_the_others_alone():
    x = matrices(4, 70, 50, "f32")
    want = P.ff_orthogonalise(x)
    x[1, 3, 4] = float("nan")
    x[2, 69, 49] = float("inf")
    got = P.ff_orthogonalise(x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3]) and not got[1:3].isfinite().any()


def test_more_matrices_than_are_worked_on_at_a_time():
    """A 1024 x 1024 matrix takes 16 MiB of the workspace, of which there is 1 GiB: 70 are two groups."""
    x = matrices(70, 1024, 1024, "bf16")
    desc = P.OrthogonaliseDesc(P.FF_BF16, 70, 1024, 1024, 5, *M.COEFFICIENTS, 1e-7)
    assert P.ff_orthogonalise_workspace_bytes(desc) < 70 * (16 << 20)
    got = P.ff_orthogonalise(x)
    # A single matrix is cut into smaller tiles.  A tile on the diagonal holds A[m][n] and A[n][m] as two sums, hi lo + lo hi + hi hi and lo hi + hi lo + hi hi, a
    # mirrored one holds one of them twice: both are within the roundings of the exact result, so they differ by twice as much, and by a step of the result's type.
    _, most = M.roundings(n64(x[0]), seeds=2)
    for i in (0, 63, 64, 69):
        alone, grouped = P.ff_orthogonalise(x[i]).double(), got[i].double()
        assert bool(((alone - grouped).abs() <= 2 * most + 2 * 2.0 ** -8 * (alone.abs() + most)).all())
    assert all(torch.equal(P.ff_orthogonalise(x), got) for _ in range(2))


def test_workspace_is_not_read_before_it_is_written():
    x = matrices(2, 50, 30, "f32")
    desc = P.OrthogonaliseDesc(P.FF_F32, 2, 50, 30, 5, *M.COEFFICIENTS, 1e-7)
    want = P.ff_orthogonalise(x)
    for fill in (0, 0xFF):
        ws = torch.full((P.ff_orthogonalise_workspace_bytes(desc),), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(P.ff_orthogonalise(x, ws=ws), want)


class Model:
    def __init__(self, shapes, param, grad, seed=0, gap=0):
        gen = torch.Generator(DEV).manual_seed(seed)

        def flat(shape, by, dtype):
            n = int(np.prod(shape))
            return (torch.randn(n + gap, generator=gen, device=DEV) * by).to(dtype)[gap:].view(shape)

        self.shapes = shapes
        kind = torch.float32 if param == "f32" else torch.bfloat16
        self.p = [flat(s, 1.0, kind) for s in shapes]
        self.master = [p.float() + flat(p.shape, 1e-4, torch.float32) for p in self.p] if param == "master" else None
        self.g = [flat(s, 0.01, DTYPES[grad]) for s in shapes]
        self.m = [flat(s, 0.005, torch.float32) for s in shapes]
        self.decay = [0.1 * (i % 3) for i in range(len(shapes))]
        self.plan = P.make_muon_plan(self.p, self.g, self.m, master=self.master, weight_decay=self.decay)

    def all(self):
        return [t.clone() for ts in (self.p, self.master or [], self.m) for t in ts]

    def check(self, run, k=1.0, **kw):
        """run() makes the step; kw: the oracle's arguments."""
        w0, m0 = [n64(t) for t in (self.master or self.p)], [n64(t) for t in self.m]
        run()
        args = {**dict(lr=0.02, beta=0.95, nesterov=True, scale="spectral", steps=5), **kw}
        for i, s in enumerate(self.shapes):
            if 0 in s:
                continue
            name = f"tensor {i} of {s}"
            decay, g = float(np.float32(self.decay[i])), n64(self.g[i])
            w, m = M.step(w0[i], g, m0[i], decay=decay, k=k, **args)
            # the clipping factor six operations, 1 - beta and the products one each, the sum one
            e_m = 12 * M.U * (np.abs(args["beta"] * m0[i]) + np.abs((1 - args["beta"]) * g * k)) + 1e-44
            assert np.all(np.abs(n64(self.m[i]) - m) <= e_m), name
            u = M.momentum(g, m0[i], args["beta"], args["nesterov"], k)[1]
            # the update's own roundings, some three times m's, pass the polynomial with a slope of 3.45 a step at most (that at 0)
            passed = 3 * np.linalg.norm(e_m) / np.linalg.norm(u) * 3.45 ** args["steps"]
            size = args["lr"] * M.step_size(args["scale"], *s)
            total, most = M.roundings(u, args["steps"])
            e_w = size * (most + passed) + 6 * M.U * (np.abs(w0[i]) + np.abs(w) + size)
            half = M.U if self.p[i].dtype == torch.float32 else 2.0 ** -8
            if self.master:
                assert np.all(np.abs(n64(self.master[i]) - w) <= e_w), name
                assert torch.equal(self.p[i], self.master[i].to(torch.bfloat16)), name
            else:
                assert np.all(np.abs(n64(self.p[i]) - w) <= e_w + half * (np.abs(w) + e_w)), name


LISTS = [[(1, 1)], [(150, 40)] * 9 + [(40, 700)] * 4 + [(33, 60)] * 3, [(64, 48), (48, 64), (130, 20), (0, 5), (20, 130), (1, 33), (33, 1), (7, 7)], [(256, 64), (64, 256), (128, 128)], [(150, 40)] + [(33, 60)] * 40 + [(100, 20)] * 25,
         [(1700, 150), (30, 20), (130, 40), (5, 5), (140, 2100)]]          # a k that is split, beside ones that are not


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "master", "bf16"])
def test_steps(param, grad):
    for shapes in LISTS:
        for gap in (0, 1):
            print(f"{param} {grad} {shapes} gap {gap}", flush=True)
            model = Model(shapes, param, grad, gap=gap)
            for _ in range(2):
                model.check(lambda: P.ff_muon_step(model.plan, 0.02))


@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(scale="rms"), dict(beta=0.0), dict(steps=2, lr=0.5), dict(lr=0.0)])
def test_step_arguments(kw):
    model = Model(LISTS[2], "f32", "f32")
    model.check(lambda: P.ff_muon_step(model.plan, **{"lr": 0.02, **kw}), **kw)


def test_clipping_and_a_norm_that_is_not_finite():
    model = Model(LISTS[2], "master", "bf16")
    norm = P.ff_grad_norm(P.make_grad_plan([g.view(-1) for g in model.g]))
    want = np.sqrt(sum((n64(g) ** 2).sum() for g in model.g))
    assert abs(norm.item() - want) <= 2 * M.U * want
    model.check(lambda: P.ff_muon_step(model.plan, 0.02, norm=norm, max_norm=0.03), k=M.clip_factor(want, 0.03))
    before = model.all()
    for bad in (float("nan"), float("inf")):
        P.ff_muon_step(model.plan, 0.02, norm=torch.tensor([bad], device=DEV), max_norm=0.03)
        assert all(torch.equal(a, b) for a, b in zip(before, model.all()))


def test_bad_gradient_stays_in_its_matrix():
    model, other = Model(LISTS[2], "f32", "f32"), Model(LISTS[2], "f32", "f32")
    model.g[2][5, 5] = float("nan")
    for m in (model, other):
        P.ff_muon_step(m.plan, 0.02)
    assert not model.p[2].isfinite().any()
    for i in range(len(model.p)):
        assert i == 2 or torch.equal(model.p[i], other.p[i])


def test_memory_around_the_matrices_is_left_alone():
    buffers = {k: torch.full((4000,), 7.0, device=DEV) for k in "pgm"}
    shapes, at, lists = [(17, 33), (9, 5), (40, 21)], 3, {k: [] for k in "pgm"}
    inside = torch.zeros(4000, dtype=torch.bool, device=DEV)
    for s in shapes:
        n = s[0] * s[1]
        for k in "pgm":
            lists[k].append(buffers[k][at:at + n].view(s))
        lists["g"][-1].copy_(torch.randn(s, device=DEV))
        inside[at:at + n] = True
        at += n + 2
    P.ff_muon_step(P.make_muon_plan(lists["p"], lists["g"], lists["m"]), 0.1)
    for k in "pgm":
        assert bool((buffers[k][~inside] == 7.0).all()), k


def test_batches_of_a_plan():
    """Matrices beyond one batch's workspace: the same as in plans of their own, up to the roundings that smaller tiles make differently (as above)."""
    shapes = [(1024, 1024)] * 66 + [(64, 32)]
    model, alone = Model(shapes, "bf16", "bf16", seed=4), Model(shapes, "bf16", "bf16", seed=4)
    w0, m0 = [n64(alone.p[0])], n64(alone.m[0])
    _, most = M.roundings(M.momentum(n64(alone.g[0]), m0, 0.95, True)[1], seeds=2)
    P.ff_muon_step(model.plan, 0.02)
    for i in (0, 63, 65, 66):
        plan = P.make_muon_plan([alone.p[i]], [alone.g[i]], [alone.m[i]], weight_decay=alone.decay[i])
        P.ff_muon_step(plan, 0.02)
        a, b = model.p[i].double(), alone.p[i].double()
        assert torch.equal(model.m[i], alone.m[i]), i
        assert bool(((a - b).abs() <= 0.02 * 2 * most * M.step_size("spectral", *shapes[i]) + 2 * 2.0 ** -8 * (a.abs() + 0.02)).all()), i
    assert not torch.equal(model.p[0].cpu().double(), torch.from_numpy(w0[0]))


def test_another_stream_and_a_graph():
    model, other = Model(LISTS[2], "master", "bf16"), Model(LISTS[2], "master", "bf16")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        P.ff_muon_step(model.plan, 0.02)
    stream.synchronize()
    P.ff_muon_step(other.plan, 0.02)
    assert all(torch.equal(a, b) for a, b in zip(model.all(), other.all()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.ff_muon_step(model.plan, 0.02)
    for turn in range(4):
        for m in (model, other):
            for i, g in enumerate(m.g):
                g.copy_(torch.randn(g.shape, generator=torch.Generator(DEV).manual_seed(10 * turn + i), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        P.ff_muon_step(other.plan, 0.02)
        assert all(torch.equal(a, b) for a, b in zip(model.all(), other.all())), turn


def test_training_operators_together():
    """Layer norm, transition, their gradients, one norm over all gradients, Muon for the matrices and AdamW for the rest: against the same in float64."""
    gen = torch.Generator(DEV).manual_seed(3)
    rows, c, f = 90, 32, 64
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    x, want = randn(rows, c), randn(rows, c)
    gamma, beta = 1 + 0.1 * randn(c), 0.1 * randn(c)
    w = [randn(f, c) / c ** 0.5, randn(f, c) / c ** 0.5, randn(c, f) / f ** 0.5]
    grads = [torch.empty_like(t) for t in (*w, gamma, beta)]
    momenta = P.muon_states(w)["m"]
    muon = P.make_muon_plan(w, grads[:3], momenta, weight_decay=0.01)
    adamw = P.make_adamw_plan([gamma, beta], grads[3:], **P.adamw_states([gamma, beta]))
    every = P.make_grad_plan(grads)
    wide = [t.double().requires_grad_() for t in (*w, gamma, beta)]

    y, _, mean, rstd = P.ff_layernorm_forward(x, gamma, beta)
    out = P.ff_gated_transition_forward(y, *w, residual=x)
    dout = 2 * (out - want) / out.numel()
    dy, *_ = P.ff_gated_transition_backward(y, *w, dout, dw_a=grads[0], dw_b=grads[1], dw_o=grads[2])
    P.ff_layernorm_backward(x, gamma, dy, mean=mean, rstd=rstd, dsum=dout, dgamma=grads[3], dbeta=grads[4])
    norm = P.ff_grad_norm(every)
    old = [n64(t) for t in w]
    P.ff_muon_step(muon, 0.02, norm=norm, max_norm=0.1)
    P.ff_adamw_step(adamw, 1, 0.01, norm=norm, max_norm=0.1)

    xd = x.double()
    unit = (xd - xd.mean(1, keepdim=True)) / (xd.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    yd = unit * wide[3] + wide[4]
    a = yd @ wide[0].t()
    loss = ((xd + (a * torch.sigmoid(a) * (yd @ wide[1].t())) @ wide[2].t() - want.double()) ** 2).mean()
    exact = torch.autograd.grad(loss, wide)
    for g, e in zip(grads, exact):
        assert (g.double() - e).norm() <= 2e-5 * e.norm()          # sums of 90 and fewer terms through four operators, 2^-24 each
    total = float(torch.cat([e.reshape(-1) for e in exact]).norm())
    assert abs(norm.item() - total) <= 2e-5 * total
    k = M.clip_factor(total, 0.1)
    for i, t in enumerate(w):
        g = exact[i].cpu().numpy()
        after, _ = M.step(old[i], g, np.zeros_like(g), lr=0.02, beta=0.95, decay=float(np.float32(0.01)), k=k)
        # the gradient's 2e-5 pass the polynomial with a slope of 3.45 in each of five steps at most
        assert np.linalg.norm(n64(t) - after) <= 0.02 * np.sqrt(2) * 2e-5 * 3.45 ** 5 + 4 * M.U * np.linalg.norm(after)
