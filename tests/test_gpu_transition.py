"""GPU parity of ff_gated_transition_forward and ff_gated_transition_backward.

Every element is held to the float64 oracle's bound of what roundings can add up to (oracle/transition.py: sums of n products n + 2 units of the sum of
magnitudes, h, da, db and results half a step of their type).
"""
import numpy as np
import pytest
import torch

import paper_2203_00854_amd as P
from oracle import transition as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: T.U, torch.bfloat16: 2.0 ** -8}
n64 = lambda t: None if t is None else t.detach().cpu().double().numpy()  # noqa: E731


class Problem:
    def __init__(self, rows, c, f, dtype, masked=False, residual=False, seed=0, gap=0):
        """gap: values in front of each tensor in its memory, so that it is aligned to no more than its type."""
        gen = torch.Generator(DEV).manual_seed(seed)

        def draw(*shape, by=1.0):
            n = int(np.prod(shape))
            flat = (torch.randn(n + gap, generator=gen, device=DEV) * by).to(DTYPES[dtype])
            return flat[gap:].view(*shape)

        self.x, self.dy = draw(rows, c), draw(rows, c)
        self.w = [draw(f, c, by=c ** -0.5), draw(f, c, by=c ** -0.5), draw(c, f, by=f ** -0.5)]
        self.residual = draw(rows, c) if residual else None
        self.mask = (torch.rand(rows, generator=gen, device=DEV) < 0.7).float() if masked else None
        if masked and rows > 1:
            self.mask[0] = 0.0
            bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device=DEV).to(self.x.dtype)
            dead = self.mask == 0
            n = int(dead.sum())
            self.x[dead] = bad[torch.arange(n, device=DEV) % 3][:, None].expand(n, c)
            self.dy[dead] = bad[torch.arange(1, n + 1, device=DEV) % 3][:, None].expand(n, c)

    def forward(self, act="silu", **kw):
        return P.ff_gated_transition_forward(self.x, *self.w, act=act, residual=self.residual, mask=self.mask, **kw)

    def backward(self, act="silu", **kw):
        return P.ff_gated_transition_backward(self.x, *self.w, self.dy, act=act, mask=self.mask, **kw)

    def check_forward(self, y, act="silu"):
        ws, x, mask, residual = [n64(w) for w in self.w], n64(self.x), n64(self.mask), n64(self.residual)
        want = T.forward(x, *ws, act, mask, residual)
        bound = T.forward_bound(x, *ws, act, HALF[self.x.dtype], mask, residual)
        off = np.abs(n64(y) - want)
        assert np.all(off <= bound), f"{(off / bound).max():.2f} of the bound at {np.unravel_index(np.argmax(off / bound), off.shape)}"

    def check_backward(self, got, act="silu", before=None):
        ws, x, dy, mask = [n64(w) for w in self.w], n64(self.x), n64(self.dy), n64(self.mask)
        want = T.backward(x, *ws, dy, act, mask)
        bound = T.backward_bound(x, *ws, dy, act, HALF[self.x.dtype], HALF[got[1].dtype], mask)
        for i, (name, g, w, e) in enumerate(zip(("dx", "dw_a", "dw_b", "dw_o"), got, want, bound)):
            if before is not None and i:
                w, e = w + before[i - 1], e + (HALF[g.dtype] + 2 * T.U) * (np.abs(before[i - 1]) + np.abs(w) + e)
            off = np.abs(n64(g) - w)
            assert np.all(off <= e), f"{name}: {(off / e).max():.2f} of the bound at {np.unravel_index(np.argmax(off / e), off.shape)}"


SIZES = [(1, 1, 1), (1, 16, 16), (3, 7, 5), (40, 64, 128), (129, 33, 70), (300, 96, 64), (257, 128, 512), (130, 256, 160), (200, 200, 312), (64, 520, 48), (300, 300, 96), (100, 32, 33), (161, 192, 256), (500, 256, 300), (400, 64, 288), (300, 512, 272),
         # few hidden channels, or many rows: rows in registers
         (2000, 250, 61), (1500, 190, 100), (700, 256, 64), (520, 192, 96), (4000, 96, 130), (9000, 128, 512),
         # with the sizes of test_gpu_transition_routes.py:
         # every tile of the other kernels
         (7000, 320, 1040), (3000, 272, 544)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,f", SIZES)
def test_forward(rows, c, f, dtype):
    for masked in (False, True):
        for residual in (False, True):
            print(f"{rows} x {c} x {f} {dtype} masked {masked} residual {residual}", flush=True)
            p = Problem(rows, c, f, dtype, masked, residual)
            p.check_forward(p.forward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,f", SIZES)
def test_backward(rows, c, f, dtype):
    for masked in (False, True):
        print(f"{rows} x {c} x {f} {dtype} masked {masked}", flush=True)
        p = Problem(rows, c, f, dtype, masked)
        p.check_backward(p.backward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "sigmoid"])
def test_activations(act, dtype):
    for rows, c, f in ((70, 64, 96), (33, 40, 20)):
        p = Problem(rows, c, f, dtype)
        for w in p.w[:2]:
            w *= 3                                  # into the activations' tails
        p.check_forward(p.forward(act), act)
        p.check_backward(p.backward(act), act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_tensors(dtype):
    for c, f in ((64, 128), (24, 40), (256, 64)):
        p = Problem(150, c, f, dtype, residual=True, gap=1)
        p.check_forward(p.forward())
        p.check_backward(p.backward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_rows_masked(dtype):
    p = Problem(50, 32, 64, dtype, residual=True)
    p.mask = torch.zeros(50, device=DEV)
    p.x.fill_(float("nan"))
    p.dy.fill_(float("inf"))
    assert torch.equal(p.forward(), p.residual)
    p.residual = None
    assert not p.forward().any()
    for t in p.backward():
        assert not t.any()


def test_no_rows():
    p = Problem(0, 32, 48, "bf16")
    assert p.forward().shape == (0, 32)
    dx, *dw = p.backward()
    assert dx.shape == (0, 32) and all(not t.any() for t in dw)
    held = [torch.ones_like(w) for w in p.w]
    p.backward(dw_a=held[0], dw_b=held[1], dw_o=held[2], accumulate=True)
    assert all(bool((t == 1).all()) for t in held)


def test_leading_shape_and_results_in_given_memory():
    p = Problem(60, 64, 96, "bf16", masked=True, residual=True)
    want = p.forward()
    shaped = lambda t: t.view(5, 12, *t.shape[1:])  # noqa: E731
    y = P.ff_gated_transition_forward(shaped(p.x), *p.w, residual=shaped(p.residual), mask=shaped(p.mask))
    assert y.shape == (5, 12, 64) and torch.equal(y.view(60, 64), want)
    held = p.residual.clone()
    again = P.ff_gated_transition_forward(p.x, *p.w, residual=held, mask=p.mask, out=held)
    assert again.data_ptr() == held.data_ptr() and torch.equal(held, want)


@pytest.mark.parametrize("dtype,grad", [("f32", torch.float32), ("bf16", torch.float32), ("bf16", torch.bfloat16)])
def test_gradients_are_added(dtype, grad):
    p = Problem(200, 48, 64, dtype, masked=True)
    gen = torch.Generator(DEV).manual_seed(5)
    held = [torch.randn(w.shape, generator=gen, device=DEV).to(grad) for w in p.w]
    before = [n64(t) for t in held]
    got = p.backward(dw_a=held[0], dw_b=held[1], dw_o=held[2], accumulate=True)
    assert all(a.data_ptr() == b.data_ptr() for a, b in zip(got[1:], held))
    p.check_backward(got, before=before)
    p.check_backward(p.backward(grad_dtype=grad))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_are_worked_on_at_a_time(dtype):
    """Rows of several chunks: each row's results are the oracle's, the weights' gradients the sums of parts."""
    c, f = 16, 2048
    rows = (512 << 20) // (f * (4 if dtype == "f32" else 2)) + 300
    p = Problem(rows, c, f, dtype)
    y, (dx, *dw) = p.forward(), p.backward(grad_dtype=torch.float32)
    part = slice(rows - 400, rows)
    q = Problem(400, c, f, dtype)
    q.w, q.x, q.dy = p.w, p.x[part].contiguous(), p.dy[part].contiguous()
    q.check_forward(y[part])
    ws, qx, qdy = [n64(w) for w in q.w], n64(q.x), n64(q.dy)
    off, bound = np.abs(n64(dx[part]) - T.backward(qx, *ws, qdy, "silu")[0]), T.backward_bound(qx, *ws, qdy, "silu", HALF[q.x.dtype], HALF[q.x.dtype])[0]
    assert np.all(off <= bound)
    total = [torch.zeros(w.shape, dtype=torch.float64, device=DEV) for w in p.w]
    for at in range(0, rows, 20000):
        q.x, q.dy = p.x[at:at + 20000].contiguous(), p.dy[at:at + 20000].contiguous()
        for t, g in zip(total, q.backward(grad_dtype=torch.float32)[1:]):
            t += g
    # Float32 sums over the rows, of terms of any sign: 8 deviations.  Fewer rows may take other kernels, whose a, b and dh differ by some 18 U each, h, da and db by e = 64 U: of
    # bfloat16 values a share 2 e / 2^-8 = 2 10^-3 then falls on the other side of a border and differs by a step, 2^-7 (2 10^-3)^(1/2) = 3.5 10^-4 of the norm.
    other = 3.5e-4 if dtype == "bf16" else 64 * T.U
    for t, g in zip(total, dw):
        assert (g - t).norm() <= (8 * T.U * rows ** 0.5 + other) * t.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,f", [(33, 20, 17), (100, 128, 32), (70, 300, 40), (2000, 250, 61)])
def test_memory_around_the_results_is_left_alone(rows, c, f, dtype):
    p = Problem(rows, c, f, dtype, masked=True, residual=True)
    around = lambda *shape: torch.full((int(np.prod(shape)) + 200,), 7.0, device=DEV, dtype=p.x.dtype)  # noqa: E731
    inside = lambda flat, *shape: flat[100:100 + int(np.prod(shape))].view(*shape)  # noqa: E731
    shapes = [(rows, c), (rows, c), (f, c), (f, c), (c, f)]
    flat = [around(*s) for s in shapes]
    y, dx, *dw = (inside(t, *s) for t, s in zip(flat, shapes))
    p.check_forward(p.forward(out=y))
    p.check_backward(p.backward(dx=dx, dw_a=dw[0], dw_b=dw[1], dw_o=dw[2]))
    for t, s in zip(flat, shapes):
        assert bool((t[:100] == 7).all()) and bool((t[100 + int(np.prod(s)):] == 7).all())


def test_wide_tokens_and_few_hidden_channels():
    """Rows of 16 KiB beside one hidden channel: as many at a time as 512 MiB hold."""
    for dtype in ("bf16", "f32"):
        p = Problem(40000, 8192, 1, dtype)
        y, (dx, *dw) = p.forward(), p.backward()
        q = Problem(50, 8192, 1, dtype)
        q.w, q.x, q.dy = p.w, p.x[-50:].contiguous(), p.dy[-50:].contiguous()
        q.check_forward(y[-50:])
        off = np.abs(n64(dx[-50:]) - T.backward(n64(q.x), *map(n64, q.w), n64(q.dy), "silu")[0])
        assert np.all(off <= T.backward_bound(n64(q.x), *map(n64, q.w), n64(q.dy), "silu", HALF[q.x.dtype], HALF[q.x.dtype])[0])
        assert all(t.isfinite().all() for t in (y, dx, *dw))


def test_equal_calls_give_equal_bits():
    p = Problem(5000, 128, 256, "bf16", masked=True, residual=True)
    y, grads = p.forward(), p.backward()
    for _ in range(3):
        assert torch.equal(p.forward(), y) and all(torch.equal(a, b) for a, b in zip(p.backward(), grads))


def test_workspace_is_not_read_before_it_is_written():
    p = Problem(300, 72, 100, "bf16", masked=True)
    desc = P.TransitionDesc(P.FF_BF16, P.FF_SILU, 72, 100, 300)
    want, grads = p.forward(), p.backward()
    for fill in (0, 0xFF):
        ws = torch.full((P.ff_gated_transition_forward_workspace_bytes(desc),), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(p.forward(ws=ws), want)
        ws = torch.full((P.ff_gated_transition_backward_workspace_bytes(desc),), fill, dtype=torch.uint8, device=DEV)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(ws=ws), grads))


def test_another_stream_and_a_graph():
    p = Problem(700, 128, 320, "bf16", masked=True, residual=True)
    y, grads = p.forward(), p.backward()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        y2, grads2 = p.forward(), p.backward()
    stream.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, grads3 = p.forward(), p.backward()
    for turn in range(4):
        p.x.copy_(torch.randn(p.x.shape, generator=torch.Generator(DEV).manual_seed(turn), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.forward(), y3) and all(torch.equal(a, b) for a, b in zip(p.backward(), grads3))


def test_gradients_against_differences():
    """Along a random direction the loss changes as the gradients say, up to third order and roundings."""
    p = Problem(48, 32, 64, "f32", masked=True)
    p.x[p.mask == 0] = 0
    p.dy[p.mask == 0] = 0
    grads = p.backward()
    gen = torch.Generator(DEV).manual_seed(9)
    live = (p.mask != 0).double()[:, None]
    for i, t in enumerate((p.x, *p.w)):
        way = torch.randn(t.shape, generator=gen, device=DEV)
        slope = (grads[i].double() * way.double() * (live if i == 0 else 1)).sum().item()
        losses, keep, h = [], t.clone(), 2.0 ** -7
        for sign in (1, -1):
            t.copy_(keep + sign * h * way)
            losses.append((p.forward().double() * p.dy.double() * live).sum().item())
        t.copy_(keep)
        # third derivatives of silu stay below 0.4, those of the products below it times the other factors: h^2 of the sizes involved; 2^-24 of 48 x 32 terms of order 1 each, over h
        size = (grads[i].double().abs() * way.double().abs()).sum().item()
        assert abs((losses[0] - losses[1]) / (2 * h) - slope) <= 2 * h * h * size + 2.0 ** -24 / h * 48 * 32
