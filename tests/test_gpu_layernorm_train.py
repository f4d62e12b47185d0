"""GPU parity of ff_layernorm_forward and ff_layernorm_backward against the float64 oracle, element by element.

Tolerances count roundings, u = 2^-24.  A sum over c <= 8192 channels passes through at most 40 additions (no more than
32 channels a lane, then a tree of lanes and wavefronts), so mean is off by at most 40 u avg|s|, and the variance by 44 u of itself
plus second order (less than 72 u with the root and the divisions).  Each further operation adds u of its operands; the store adds half a step of the output type.  Sums over
rows: at most D additions, D u sum|terms|, plus what the terms themselves are off by.
"""
import numpy as np
import pytest
import torch

import paper_2203_00854_amd as P
from oracle import layernorm_train as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def half_step(dtype):
    return torch.finfo(DT[dtype]).eps / 2


def make(rows, c, dtype, seed, offset=0.5, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    t = {"x": r(rows, c) * scale + offset * r(rows, 1), "residual": r(rows, c), "dy": r(rows, c), "dsum": r(rows, c), "gamma": 1 + 0.3 * r(c), "beta": 0.3 * r(c)}
    return {k: v.to(DT[dtype]) for k, v in t.items()}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def up(t, shift=0):
    """On the GPU; shift: values between an allocation's start and the tensor's."""
    if not shift:
        return t.to(DEV)
    room = torch.zeros(t.numel() + shift, dtype=t.dtype, device=DEV)
    room[shift:] = t.reshape(-1).to(DEV)
    return room[shift:].view(t.shape)


def bounds(s, gamma, beta, eps=EPS):
    """What mean, rstd (relative), the normalised value and y may be off by, before the store."""
    y, mean, rstd = O.forward(s, gamma, beta, eps)
    e_mean = 40 * U * np.abs(s).mean(1) + U * np.abs(mean)
    e_rstd = 72 * U + (e_mean * rstd) ** 2
    unit = (s - mean[:, None]) * rstd[:, None]
    e_unit = (rstd * e_mean)[:, None] + (e_rstd[:, None] + 3 * U) * np.abs(unit)
    e_y = np.abs(gamma) * (e_unit + U * np.abs(unit)) + 2 * U * (np.abs(y) + np.abs(beta))
    return y, mean, rstd, unit, e_mean, e_rstd, e_unit, e_y


def check(name, got, want, tol):
    off = np.abs(got - want)
    print(f"{name}: worst share of the tolerance {float((off / np.maximum(tol, 1e-300)).max()) if off.size else 0:.3f}", flush=True)
    assert np.isfinite(got).all(), name
    assert np.all(off <= tol), (name, float((off - tol).max()))


def check_forward(t, dtype, out, residual):
    y, kept, mean, rstd = out
    s = t["x"]
    if residual:
        s = (t["x"].float() + t["residual"].float()).to(DT[dtype])
        assert torch.equal(kept.cpu(), s)
    else:
        assert kept is None
    want, m, r, _, e_mean, e_rstd, _, e_y = bounds(f64(s), f64(t["gamma"]), f64(t["beta"]))
    check("y", f64(y), want, e_y + half_step(dtype) * (np.abs(want) + e_y))
    if mean is not None:
        check("mean", f64(mean), m, e_mean + U * np.abs(m))
        check("rstd", f64(rstd), r, (e_rstd + U) * r)


def check_backward(s, t, dtype, out, dsum, base=None):
    dx, dgamma, dbeta = out
    s64, g64, dy = f64(s), f64(t["gamma"]), f64(t["dy"])
    rows, c = s64.shape
    want = O.backward(s64, g64, dy, EPS, f64(t["dsum"]) if dsum else None)
    _, _, rstd, unit, _, e_rstd, e_unit, _ = bounds(s64, g64, np.zeros(c))
    h = dy * g64
    a, b = h.mean(1, keepdims=True), (h * unit).mean(1, keepdims=True)
    e_a = 42 * U * np.abs(h).mean(1, keepdims=True)
    e_b = 44 * U * np.abs(h * unit).mean(1, keepdims=True) + (np.abs(h) * e_unit).mean(1, keepdims=True)
    size = np.abs(h) + np.abs(a) + np.abs(unit * b)
    e_dx = rstd[:, None] * (4 * U * size + e_a + np.abs(unit) * e_b + e_unit * np.abs(b)) + (e_rstd[:, None] + 2 * U) * rstd[:, None] * size
    if dsum:
        e_dx = e_dx + U * (np.abs(want[0]) + np.abs(f64(t["dsum"])))
    check("dx", f64(dx), want[0], e_dx + half_step(dtype) * (np.abs(want[0]) + e_dx))
    depth = min(rows, 1200) + 2
    add = (0.0, 0.0) if base is None else base
    check("dgamma", f64(dgamma), want[1] + add[0], depth * U * np.abs(dy * unit).sum(0) + (np.abs(dy) * e_unit).sum(0) + U * np.abs(want[1] + add[0]) + 1e-38)
    check("dbeta", f64(dbeta), want[2] + add[1], depth * U * np.abs(dy).sum(0) + U * np.abs(want[2] + add[1]) + 1e-38)


# rows, c: one row and one channel, channels below and between whole vectors and lanes, every number of pieces a lane can hold, rows for a few and for many blocks
SHAPES = [(1, 1), (7, 1), (5, 2), (3, 3), (64, 5), (9, 7), (1, 8), (33, 16), (257, 24), (2049, 32), (100, 40), (1, 64), (513, 64), (70, 96), (19, 100), (300, 128), (12, 173),
          (40, 256), (65, 257), (31, 384), (17, 500), (18, 512), (9, 513), (11, 768), (6, 1000), (5, 1024), (7, 1025), (4, 2048), (3, 2049), (5, 4093), (3, 4096),
          (2, 6000), (3, 8191), (2, 8192)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
def test_forward_and_backward(rows, c, dtype):
    t = make(rows, c, dtype, seed=rows * 10007 + c)
    for residual in (False, True):
        for saved in (True, False):
            print(f"rows {rows} c {c} {dtype} residual {residual} saved {saved}", flush=True)
            d = {k: up(v) for k, v in t.items()}
            out = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], residual=d["residual"] if residual else None, eps=EPS, stats=saved)
            torch.cuda.synchronize()
            check_forward(t, dtype, out, residual)
            s = out[1] if residual else d["x"]
            grads = P.ff_layernorm_backward(s, d["gamma"], d["dy"], mean=out[2], rstd=out[3], dsum=d["dsum"] if residual else None, eps=EPS)
            torch.cuda.synchronize()
            check_backward(s.cpu(), t, dtype, grads, residual)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(50_000, 64), (20_000, 128), (9920, 173), (6000, 384)])
def test_many_rows(rows, c, dtype):
    t = make(rows, c, dtype, seed=c)
    d = {k: up(v) for k, v in t.items()}
    out = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], eps=EPS)
    check_forward(t, dtype, out, False)
    grads = P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], mean=out[2], rstd=out[3], eps=EPS)
    check_backward(t["x"], t, dtype, grads, False)
    again = P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], mean=out[2], rstd=out[3], eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))        # the order of the sums is fixed


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(70_001, 1), (70_001, 3), (40_000, 8), (30_011, 12), (30_011, 16), (20_000, 24), (20_000, 31)])
def test_short_rows(rows, c, dtype):
    """Teams of one to four lanes, in one block and in many."""
    for n in (rows, 1023):
        t = make(n, c, dtype, seed=c)
        d = {k: up(v) for k, v in t.items()}
        out = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], residual=d["residual"], eps=EPS)
        check_forward(t, dtype, out, True)
        for saved in (True, False):
            grads = P.ff_layernorm_backward(out[1], d["gamma"], d["dy"], mean=out[2] if saved else None, rstd=out[3] if saved else None, dsum=d["dsum"], eps=EPS)
            check_backward(out[1].cpu(), t, dtype, grads, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [24, 128, 173, 1000, 3000])
@pytest.mark.parametrize("shift", [1, 3, 4])
def test_tensors_at_any_offset(c, dtype, shift):
    t = make(37, c, dtype, seed=shift)
    d = {k: up(v, shift + (i % 2)) for i, (k, v) in enumerate(t.items())}
    for residual in (False, True):
        out = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], residual=d["residual"] if residual else None, eps=EPS, out=up(torch.zeros_like(t["x"]), shift))
        check_forward(t, dtype, out, residual)
        s = out[1] if residual else d["x"]
        grads = P.ff_layernorm_backward(s, d["gamma"], d["dy"], dsum=d["dsum"] if residual else None, eps=EPS, dx=up(torch.zeros_like(t["x"]), shift))
        check_backward(s.cpu(), t, dtype, grads, residual)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [1, 100, 256, 1500])
def test_in_place_and_guarded(c, dtype):
    """sum over x or residual, dx over dy or dsum; what lies around the outputs stays."""
    t = make(45, c, dtype, seed=c + 1)
    n = 45 * c

    def guarded(src):
        room = torch.full((n + 64,), 7.0, dtype=DT[dtype], device=DEV)
        view = room[32:32 + n].view(45, c)
        if src is not None:
            view.copy_(src.to(DEV))
        return room, view

    for over in ("x", "residual"):
        (rx, x), (rr, res), (ry, y) = guarded(t["x"]), guarded(t["residual"]), guarded(None)
        out = P.ff_layernorm_forward(x, up(t["gamma"]), up(t["beta"]), residual=res, eps=EPS, sum_out=x if over == "x" else res, out=y)
        check_forward(t, dtype, out, True)
        for room in (rx, rr, ry):
            assert (room[:32] == 7).all() and (room[32 + n:] == 7).all()
    for over in ("dy", "dsum"):
        (ry, dy), (rs, dsum) = guarded(t["dy"]), guarded(t["dsum"])
        grads = P.ff_layernorm_backward(up(t["x"]), up(t["gamma"]), dy, dsum=dsum, eps=EPS, dx=dy if over == "dy" else dsum)
        check_backward(t["x"], t, dtype, grads, True)
        for room in (ry, rs):
            assert (room[:32] == 7).all() and (room[32 + n:] == 7).all()


def test_accumulation_and_no_rows():
    t = make(30, 64, "f32", seed=3)
    d = {k: up(v) for k, v in t.items()}
    dgamma, dbeta = torch.full((64,), 2.0, device=DEV), torch.full((64,), -3.0, device=DEV)
    out = P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], eps=EPS, dgamma=dgamma, dbeta=dbeta, accumulate=True)
    check_backward(t["x"], t, "f32", out, False, base=(2.0, -3.0))
    none = torch.empty(0, 64, device=DEV)
    kept = dgamma.clone()
    P.ff_layernorm_backward(none, d["gamma"], none, eps=EPS, dgamma=dgamma, dbeta=dbeta, accumulate=True)
    assert torch.equal(kept, dgamma)
    _, dg, db = P.ff_layernorm_backward(none, d["gamma"], none, eps=EPS, dgamma=dgamma, dbeta=dbeta)
    assert (dg == 0).all() and (db == 0).all()
    y, _, mean, _ = P.ff_layernorm_forward(none, d["gamma"], d["beta"])
    assert y.shape == (0, 64) and mean.shape == (0,)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [16, 128, 173, 1100])
def test_values_that_are_not_finite_stay_in_their_row(c, dtype):
    t = make(64, c, dtype, seed=9)
    d = {k: up(v) for k, v in t.items()}
    clean = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], eps=EPS)
    dirty = d["x"].clone()
    dirty[5, 3] = float("nan")
    dirty[9, c - 1] = float("inf")
    y = P.ff_layernorm_forward(dirty, d["gamma"], d["beta"], eps=EPS)[0]
    dx = P.ff_layernorm_backward(dirty, d["gamma"], d["dy"], eps=EPS)[0]
    want_dx = P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], eps=EPS)[0]
    keep = torch.ones(64, dtype=torch.bool, device=DEV)
    keep[5] = keep[9] = False
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(dx[keep], want_dx[keep])
    assert y[~keep].isnan().all() and dx[~keep].isnan().all()


def test_constant_rows_and_large_means():
    """No variance: rstd is 1 / sqrt(eps), y is beta.  A mean of 1000 deviations costs what the bound says and no more."""
    gamma, beta = torch.ones(128, device=DEV), torch.full((128,), 0.25, device=DEV)
    y, _, mean, rstd = P.ff_layernorm_forward(torch.full((5, 128), 3.0, device=DEV), gamma, beta, eps=1e-5)
    assert (y == 0.25).all() and (mean == 3).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
    t = make(50, 128, "f32", seed=4, offset=1000.0)
    d = {k: up(v) for k, v in t.items()}
    out = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], eps=EPS)
    check_forward(t, "f32", out, False)
    check_backward(t["x"], t, "f32", P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], eps=EPS), False)


def test_gradient_against_differences():
    """The gradient against differences of the forward kernel's own outputs.  Along a direction of unit entries the loss changes by
    its slope times the step up to third order: (step^2 / 6) times a third derivative of order sum|dy|, and the outputs' rounding,
    10 u max|y| sum|dy| / step."""
    t = make(6, 128, "f32", seed=12)
    d = {k: up(v) for k, v in t.items()}
    dx, dgamma, dbeta = P.ff_layernorm_backward(d["x"], d["gamma"], d["dy"], eps=EPS)
    gen = torch.Generator(DEV).manual_seed(1)
    step = 2.0 ** -7
    for which, grad in (("x", dx), ("gamma", dgamma), ("beta", dbeta)):
        along = torch.randint(0, 2, d[which].shape, generator=gen, device=DEV) * 2.0 - 1
        ends = []
        for sign in (1, -1):
            a = {**d, which: d[which] + sign * step * along}
            ends.append((P.ff_layernorm_forward(a["x"], a["gamma"], a["beta"], eps=EPS)[0].double() * d["dy"].double()).sum())
        slope, want = (ends[0] - ends[1]) / (2 * step), (grad.double() * along.double()).sum()
        weight = d["dy"].abs().sum().item()
        assert abs(slope.item() - want.item()) <= weight * (step ** 2 + 40 * U / step), which


def test_captured_into_a_graph_and_on_another_stream():
    t = make(2000, 128, "bf16", seed=6)
    d = {k: up(v) for k, v in t.items()}
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    names = ("y", "sum", "dx", "dgamma", "dbeta")
    buf = {k: torch.empty_like(d["x"]) for k in names[:3]} | {k: torch.empty(128, device=DEV) for k in names[3:]}

    def work():
        P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], residual=d["residual"], eps=EPS, stats=False, out=buf["y"], sum_out=buf["sum"])
        P.ff_layernorm_backward(buf["sum"], d["gamma"], d["dy"], dsum=d["dsum"], eps=EPS, dx=buf["dx"], dgamma=buf["dgamma"], dbeta=buf["dbeta"], ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    gen = torch.Generator(DEV).manual_seed(2)
    for _ in range(4):
        d["x"].copy_(torch.randn(2000, 128, generator=gen, device=DEV))
        d["dy"].copy_(torch.randn(2000, 128, generator=gen, device=DEV))
        work()
        torch.cuda.synchronize()
        eager = {k: v.clone() for k, v in buf.items()}
        for v in buf.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(buf[k], eager[k]), k


def test_rows_beyond_32_bit_offsets():
    """Values past 2^31 and bytes past 2^32: the last rows are those of a small call."""
    rows, c = (1 << 24) + 3, 144
    x = torch.empty(rows, c, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(DEV).manual_seed(5)
    x.fill_(0.0)
    tail = torch.randn(64, c, generator=gen, device=DEV).to(torch.bfloat16)
    x[-64:] = tail
    x[:64] = tail.flip(0)
    gamma, beta = torch.rand(c, generator=gen, device=DEV).to(torch.bfloat16), torch.rand(c, generator=gen, device=DEV).to(torch.bfloat16)
    y, _, mean, rstd = P.ff_layernorm_forward(x, gamma, beta, eps=EPS)
    small = P.ff_layernorm_forward(tail, gamma, beta, eps=EPS)
    assert torch.equal(y[-64:], small[0]) and torch.equal(mean[-64:], small[2]) and torch.equal(y[:64], small[0].flip(0))
    assert (y[64:-64:1_000_003] == beta).all()
    dy = torch.zeros_like(x)
    dy[-64:] = tail
    dx, dgamma, dbeta = P.ff_layernorm_backward(x, gamma, dy, mean=mean, rstd=rstd, eps=EPS)
    want = P.ff_layernorm_backward(tail, gamma, tail, eps=EPS)
    assert torch.equal(dx[-64:], want[0]) and (dx[:-64:1_000_003] == 0).all()
    assert torch.allclose(dgamma, want[1], rtol=1e-5, atol=1e-4) and torch.allclose(dbeta, want[2], rtol=1e-5, atol=1e-4)


def test_refused_tensors():
    x, g = torch.randn(20, 64, device=DEV), torch.ones(64, device=DEV)
    cases = [(dict(x=x.t().contiguous().t()), ValueError), (dict(x=x.half()), TypeError), (dict(gamma=g[:32]), ValueError), (dict(beta=g.bfloat16()), TypeError),
             (dict(residual=x[:10]), ValueError), (dict(out=x), P.FFError), (dict(sum_out=x), ValueError), (dict(residual=x.bfloat16()), TypeError),
             (dict(eps=-1.0), P.FFError), (dict(gamma=g.cpu()), ValueError), (dict(out=torch.empty(20, 65, device=DEV)), ValueError)]
    for kw, error in cases:
        with pytest.raises(error):
            P.ff_layernorm_forward(**{**dict(x=x, gamma=g, beta=g), **kw})
    _, _, mean, rstd = P.ff_layernorm_forward(x, g, g)
    cases = [(dict(dy=x[:, :32]), ValueError), (dict(mean=mean), P.FFError), (dict(mean=mean[:5], rstd=rstd[:5]), ValueError), (dict(dsum=x.bfloat16()), TypeError),
             (dict(accumulate=True), ValueError), (dict(dx=x), P.FFError), (dict(ws=torch.empty(8, dtype=torch.uint8, device=DEV)), P.FFError),
             (dict(dgamma=g.bfloat16(), dbeta=g.clone()), TypeError), (dict(dgamma=g, dbeta=g.clone()), P.FFError)]
    for kw, error in cases:
        with pytest.raises(error):
            P.ff_layernorm_backward(**{**dict(s=x, gamma=g, dy=x.clone()), **kw})


def test_leading_axes():
    """[n_a, n_b, c] as the modules have it: statistics of that shape without the channels."""
    x = torch.randn(6, 10, 64, device=DEV)
    g, b = torch.rand(64, device=DEV), torch.rand(64, device=DEV)
    y, _, mean, rstd = P.ff_layernorm_forward(x, g, b)
    flat = P.ff_layernorm_forward(x.view(60, 64), g, b)
    assert mean.shape == (6, 10) and torch.equal(y.view(60, 64), flat[0]) and torch.equal(rstd.view(60), flat[3])
    dx, dgamma, _ = P.ff_layernorm_backward(x, g, y, mean=mean, rstd=rstd)
    want = P.ff_layernorm_backward(x.view(60, 64), g, y.view(60, 64), mean=flat[2], rstd=flat[3])
    assert torch.equal(dx.view(60, 64), want[0]) and torch.equal(dgamma, want[1])


@pytest.mark.parametrize("dtype,rows,c", [("bf16", 500_000, 128), ("bf16", 500_000, 100), ("f32", 150_000, 173), ("bf16", 90_000, 1100), ("f32", 30_000, 2000)])
def test_inputs_beyond_the_caches(dtype, rows, c):
    """Sizes whose inputs are loaded past the caches: rows from all over the tensor against the oracle, sums over all rows in float64,
    results in place as well."""
    gen = torch.Generator(DEV).manual_seed(c)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(DT[dtype])  # noqa: E731
    d = {"x": randn(rows, c), "residual": randn(rows, c), "dy": randn(rows, c), "dsum": randn(rows, c), "gamma": randn(c), "beta": randn(c)}
    assert 160e6 < 2 * d["x"].numel() * d["x"].element_size() < 1e9
    some = torch.cat([torch.arange(40), torch.arange(0, rows, 9973), torch.arange(rows - 40, rows)]).to(DEV)
    part = {k: (v[some] if v.dim() == 2 else v).cpu() for k, v in d.items()}
    y, s, mean, rstd = P.ff_layernorm_forward(d["x"], d["gamma"], d["beta"], residual=d["residual"], eps=EPS)
    check_forward(part, dtype, (y[some], s[some], mean[some], rstd[some]), True)
    del y
    for saved in (True, False):
        kw = dict(mean=mean, rstd=rstd) if saved else {}
        dx, dgamma, dbeta = P.ff_layernorm_backward(s, d["gamma"], d["dy"], dsum=d["dsum"], eps=EPS, **kw)
        u = (s.double() - mean.double()[:, None]) * rstd.double()[:, None]
        terms = d["dy"].double() * u
        # at most 1200 additions, and the terms' own error: what mean and rstd are off by (test's head) and two operations
        size = terms.abs().sum(0)
        off = (1200 + 80) * U * size + (d["dy"].double().abs() * (45 * U * s.double().abs().mean(1) * rstd.double())[:, None]).sum(0)
        assert ((dgamma.double() - terms.sum(0)).abs() <= off).all()
        assert ((dbeta.double() - d["dy"].double().sum(0)).abs() <= 1200 * U * d["dy"].double().abs().sum(0)).all()
        del u, terms
        small = P.ff_layernorm_backward(s[some], d["gamma"], d["dy"][some], dsum=d["dsum"][some], eps=EPS, **{k: v[some] for k, v in kw.items()})
        check_backward(s[some].cpu(), part, dtype, (dx[some], small[1], small[2]), True)
        over = d["dy"].clone() if saved else d["dsum"].clone()
        args = dict(dy=over, dsum=d["dsum"]) if saved else dict(dy=d["dy"], dsum=over)
        again = P.ff_layernorm_backward(s, d["gamma"], eps=EPS, dx=over, **args, **kw)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta)


@pytest.mark.parametrize("dtype,rows,c", [("bf16", 60_001, 128), ("bf16", 40_000, 173), ("bf16", 90_011, 24), ("bf16", 12_003, 1000), ("bf16", 70_001, 3),
                                          ("f32", 1_050_001, 128), ("f32", 1_050_001, 125)])
def test_backward_with_the_next_row_on_its_way(dtype, rows, c):
    """Many turns of rows a block with saved statistics: rows from all over the tensor against the oracle, sums over all rows in float64, in place as well."""
    gen = torch.Generator(DEV).manual_seed(c + 1)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(DT[dtype])  # noqa: E731
    d = {"x": randn(rows, c), "dy": randn(rows, c), "dsum": randn(rows, c), "gamma": randn(c), "beta": randn(c)}
    size = 2 * d["x"].numel() * d["x"].element_size()
    assert size < 160e6 if dtype == "bf16" else size > 1e9
    some = torch.cat([torch.arange(40), torch.arange(0, rows, 997), torch.arange(rows - 40, rows)]).to(DEV)
    part = {k: (v[some] if v.dim() == 2 else v).cpu() for k, v in d.items()}
    x, gamma, dy = d["x"], d["gamma"], d["dy"]
    _, _, mean, rstd = P.ff_layernorm_forward(x, gamma, d["beta"], eps=EPS)
    terms = dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])
    # at most 1200 additions, and the terms' own error: what mean and rstd are off by (test's head) and two operations
    off = (1200 + 80) * U * terms.abs().sum(0) + (dy.double().abs() * (45 * U * x.double().abs().mean(1) * rstd.double())[:, None]).sum(0)
    want, off_b = terms.sum(0), 1200 * U * dy.double().abs().sum(0)
    del terms
    for dsum in (None, d["dsum"]):
        kw = dict(mean=mean, rstd=rstd, dsum=dsum, eps=EPS)
        dx, dgamma, dbeta = P.ff_layernorm_backward(x, gamma, dy, **kw)
        assert ((dgamma.double() - want).abs() <= off).all()
        assert ((dbeta.double() - dy.double().sum(0)).abs() <= off_b).all()
        small = P.ff_layernorm_backward(x[some], gamma, dy[some], mean=mean[some], rstd=rstd[some], dsum=None if dsum is None else dsum[some], eps=EPS)
        check_backward(part["x"], part, dtype, (dx[some], small[1], small[2]), dsum is not None)
        over = dy.clone()
        again = P.ff_layernorm_backward(x, gamma, over, dx=over, **kw)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma) and torch.equal(again[2], dbeta)


@pytest.mark.parametrize("dtype,rows,c,own", [("f32", 16, 256, 1), ("bf16", 16, 512, 1), ("f32", 61, 200, 4), ("f32", 300, 2048, 1), ("f32", 1000, 1100, 2),
                                              ("bf16", 700, 1500, 1), ("f32", 4096, 256, 1), ("bf16", 8000, 300, 2)])
def test_sums_over_rows_lose_nothing_between_wavefronts_and_blocks(dtype, rows, c, own):
    """A row of 2^24 beside rows of 1, which a float32 sum that has reached 2^24 does not take in.  Only a wavefront's (or, of long rows, a block's) own rows,
    here `own` of them at most, are added up in float32, so that no more than the ones beside the large row can be lost; a block's sum and
    the result are rounded once each."""
    x, dy = torch.randn(rows, c, device=DEV).to(DT[dtype]), torch.ones(rows, c, device=DEV, dtype=DT[dtype])
    dy[rows // 2] = 2.0 ** 24
    want = 2.0 ** 24 + rows - 1
    gamma = torch.ones(c, device=DEV, dtype=DT[dtype])
    _, _, dbeta = P.ff_layernorm_backward(x, gamma, dy, eps=EPS)
    off = (dbeta.double() - want).abs().max().item()
    print(f"off by {off}", flush=True)
    assert off <= own - 1 + 2 * U * want
    _, _, dbeta = P.ff_layernorm_backward(x, gamma, dy, eps=EPS, dgamma=torch.zeros(c, device=DEV), dbeta=torch.full((c,), 5.0, device=DEV), accumulate=True)
    assert (dbeta.double() - (want + 5)).abs().max().item() <= own - 1 + 2 * U * (want + 5)
