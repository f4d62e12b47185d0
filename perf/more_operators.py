"""Timing cases of a gated transition and of the optimiser for its matrices: the transition's forward and backward pass,
orthogonalising an update by Newton-Schulz products, and the Muon step over all matrices of a model.

listed() names twelve passes from the smallest call to the largest, draw() gives further ones of the same ranges.  Shapes are those of
inputs.py and bench.py (initial-training crop 128 x 256, pairs at 701 and 2048 residues, rows of odd channel counts) with hidden
layers of two to four times the channels; the optimiser's matrices are the weights of ff.h's modules and of both transitions in up to
48 Evoformer blocks, or ragged lists.  Where `own` is false run() computes the operators in elementary torch operations.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7                                     # beside the norm of an update
HYPER = {"lr": 0.02, "beta": 0.95}
DECAY = 0.01


# --------------------------------------------------------------------------------------------------- the cases
def _transition(name, op, rows, c, f, dtype, act="silu", residual=False, masked=False):
    return {"name": name, "op": op, "rows": rows, "c": c, "f": f, "dtype": dtype, "act": act, "residual": residual, "masked": masked}


def _orthogonalise(name, count, rows, cols, dtype, steps=5):
    return {"name": name, "op": "orthogonalise", "count": count, "rows": rows, "cols": cols, "dtype": dtype, "steps": steps}


def _muon(name, layout, count, most, grad, param, nesterov, scale):
    return {"name": name, "op": "muon", "layout": layout, "count": count, "most": most, "grad": grad, "param": param, "nesterov": nesterov, "scale": scale}


def listed():
    return [
        # one residue axis of a toy crop: the smallest call, where launches count
        _transition("transition_f32_40x64", "forward", 40, 64, 128, "f32"),
        # the MSA representation of the initial-training crop, closed by the residual sum
        _transition("transition_bf16_128x256x256_sum", "forward", 128 * 256, 256, 1024, "bf16", residual=True),
        # 64 sequences x 155 residues, channels that fill no whole vector
        _transition("transition_f32_9920x173", "forward", 64 * 155, 173, 692, "f32", act="gelu"),
        # the pair representation at 2048 residues with the residual sum: the largest call
        _transition("transition_bf16_2048x2048x128_sum", "forward", 2048 * 2048, 128, 512, "bf16", residual=True),
        # the smallest gradient
        _transition("transition_backward_f32_40x64", "backward", 40, 64, 128, "f32"),
        # the gradient at the MSA representation of the initial-training crop
        _transition("transition_backward_bf16_128x256x256", "backward", 128 * 256, 256, 1024, "bf16"),
        # the pair representation of a protein of odd length, in a batch that pads it
        _transition("transition_backward_bf16_701x701x128", "backward", 701 * 701, 128, 512, "bf16", masked=True),
        # 60 sequences x 300 residues with odd channels
        _transition("transition_backward_f32_18000x173", "backward", 60 * 300, 173, 692, "f32", act="sigmoid"),
        # one projection of a small module: the smallest update
        _orthogonalise("orthogonalise_f32_128x64", 1, 128, 64, "f32"),
        # the update of one wide hidden layer
        _orthogonalise("orthogonalise_bf16_4096x1024", 1, 4096, 1024, "bf16"),
        # a dozen matrices of no common size
        _muon("muon_12_ragged", "ragged", 12, 700, "f32", "f32", False, "rms"),
        # the step of the whole stack: 1968 matrices, bfloat16 weights and gradients, float32 master weights
        _muon("muon_48_blocks_master", "evoformer", 48, 0, "bf16", "master", True, "spectral"),
    ]


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(("forward", "forward", "backward", "backward", "orthogonalise", "muon"))
    dtype = rng.choice(("f32", "bf16"))
    if op in ("forward", "backward"):
        c = rng.choice((32, 64, 128, 256, 384, spread(8, 1024), spread(8, 300)))
        f = rng.choice((2 * c, 4 * c, 4 * c, spread(8, 4096)))
        most = {"forward": 2.7e11, "backward": 8e10}[op] / (8 if dtype == "f32" else 1)
        rows = spread(1, max(1, min(2_000_000, int(most / (c * f)))))
        return {"op": op, "rows": rows, "c": c, "f": f, "dtype": dtype, "act": rng.choice(("silu", "silu", "gelu", "sigmoid")),
                "residual": op == "forward" and rng.random() < 0.5, "masked": rng.random() < 0.4}
    if op == "orthogonalise":
        rows, cols = spread(1, 2048), spread(1, 2048)
        n, m = min(rows, cols), max(rows, cols)
        return {"op": op, "count": spread(1, max(1, min(64, int(4e9 / (3 * n * n * m + n ** 3))))), "rows": rows, "cols": cols, "dtype": dtype, "steps": rng.choice((5, 5, 3))}
    more = {"grad": dtype, "param": rng.choice(("f32", "master", "bf16")), "nesterov": rng.random() < 0.5, "scale": rng.choice(("spectral", "rms"))}
    if rng.random() < 0.5:
        return {"op": op, "layout": "evoformer", "count": spread(1, 47), "most": 0, **more}
    return {"op": op, "layout": "ragged", "count": spread(1, 24), "most": spread(16, 1024), **more}


def _shapes(case):
    """{shape: how many} of the optimiser's matrices."""
    if case["layout"] == "ragged":
        rng = random.Random(case["count"] * 1_000_003 + case["most"])
        shapes = [(max(1, int(case["most"] ** rng.random())), max(1, int(case["most"] * rng.random()))) for _ in range(case["count"])]
    else:
        m, z, heads, tri = 256, 128, 8, 4
        row = [(m, m)] * 5 + [(heads, z)]
        col = [(m, m)] * 5
        triangle = [(z, z)] * 5 + [(tri, z)]
        update = [(z, z)] * 6
        transitions = [(4 * m, m)] * 2 + [(m, 4 * m)] + [(4 * z, z)] * 2 + [(z, 4 * z)]
        shapes = (row + col + triangle * 2 + update * 2 + transitions) * case["count"]
    return {s: shapes.count(s) for s in sorted(set(shapes), reverse=True)}


# --------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
    if case["op"] in ("forward", "backward"):
        return _prepare_transition(case, randn, gen)
    if case["op"] == "orthogonalise":
        return {"case": case, "x": _gradients(randn, case["count"], case["rows"], case["cols"]).to(DTYPES[case["dtype"]])}
    return _prepare_muon(case, randn)


def _prepare_transition(case, randn, gen):
    rows, c, f, t = case["rows"], case["c"], case["f"], DTYPES[case["dtype"]]
    wide = lambda: randn(rows, c).to(t)  # noqa: E731
    s = {"case": case, "x": wide(), "w_a": (randn(f, c) / c ** 0.5).to(t), "w_b": (randn(f, c) / c ** 0.5).to(t), "w_o": (randn(c, f) / f ** 0.5).to(t)}
    s["mask"] = (torch.rand(rows, generator=gen, device=DEV) < 0.9).float() if case["masked"] else None
    if case["op"] == "backward":
        s["dy"] = wide()
    else:
        s["residual"] = wide() if case["residual"] else None
    return s


def _gradients(randn, count, rows, cols):
    """Sums over few tokens above noise, as gradients of weights are: singular values that fall by some powers of ten, of any common size."""
    k = min(8, rows, cols)
    size = torch.exp(randn(count, 1, 1) - 5.0)
    return size * (randn(count, rows, k) @ (randn(count, k, cols) * torch.exp(-torch.arange(k, device=DEV) / 2.0)[:, None]) + 0.2 * randn(count, rows, cols))


def _prepare_muon(case, randn):
    shapes, t = _shapes(case), DTYPES[case["grad"]]
    s = {"case": case, "g": [], "p": [], "master": [], "m": []}              # matrices of one shape lie together
    for (rows, cols), n in shapes.items():
        s["g"].append(_gradients(randn, n, rows, cols).to(t))
        s["m"].append(0.5 * _gradients(randn, n, rows, cols))
        w = randn(n, rows, cols) / cols ** 0.5
        s["p"].append(w if case["param"] == "f32" else w.to(torch.bfloat16))
        if case["param"] == "master":
            s["master"].append(w)
    if own:                                   # a program that trains keeps the plan of its matrices
        import paper_2203_00854_amd as P
        each = lambda k: [t for group in s[k] for t in group.unbind(0)]  # noqa: E731
        s["plan"] = P.make_muon_plan(each("p"), each("g"), each("m"), master=each("master") or None, weight_decay=DECAY)
    return s


# --------------------------------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _gate(act, a):
    """act(a) and its derivative."""
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(a / math.sqrt(2)))
        return a * phi, phi + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-a))
    if act == "sigmoid":
        return sig, sig * (1 - sig)
    return a * sig, sig * (1 + a * (1 - sig))


def _live(t, mask):
    """What a masked row holds takes no part, whatever it is."""
    return t.float() if mask is None else torch.where(mask[:, None] != 0, t.float(), 0.0)


def _plain_forward(s):
    x = _live(s["x"], s["mask"])
    a, b = x @ s["w_a"].float().t(), x @ s["w_b"].float().t()
    y = (_gate(s["case"]["act"], a)[0] * b) @ s["w_o"].float().t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_backward(s):
    t = s["x"].dtype
    x, dy = _live(s["x"], s["mask"]), _live(s["dy"], s["mask"])
    w_a, w_b, w_o = s["w_a"].float(), s["w_b"].float(), s["w_o"].float()
    a, b = x @ w_a.t(), x @ w_b.t()
    gate, slope = _gate(s["case"]["act"], a)
    dh = dy @ w_o
    da, db = dh * b * slope, dh * gate
    return {"dx": (da @ w_a + db @ w_b).to(t), "dw_a": (da.t() @ x).to(t), "dw_b": (db.t() @ x).to(t), "dw_o": (dy.t() @ (gate * b)).to(t)}


def _newton_schulz(g, steps):
    """Batches [n, rows, cols] of float32 matrices, orthogonalised on their shorter side."""
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = (x.double() / (norm + EPS)).float()
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        gram = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_orthogonalise(s):
    return _newton_schulz(s["x"].float(), s["case"]["steps"]).contiguous().to(s["x"].dtype)


def _step_scale(kind, rows, cols):
    return max(1.0, rows / cols) ** 0.5 if kind == "spectral" else 0.2 * max(rows, cols) ** 0.5


def _plain_muon(s):
    case, beta = s["case"], HYPER["beta"]
    for i, g in enumerate(s["g"]):
        now = (1 - beta) * g.float()
        s["m"][i].copy_(beta * s["m"][i] + now)
        update = _newton_schulz(beta * s["m"][i] + now if case["nesterov"] else s["m"][i], 5)
        w = (s["master"][i] if s["master"] else s["p"][i]).float()
        w = w - HYPER["lr"] * (DECAY * w + _step_scale(case["scale"], g.shape[1], g.shape[2]) * update)
        s["p"][i].copy_(w)
        if s["master"]:
            s["master"][i].copy_(w)
    return {"p": s["p"], "master": s["master"], "m": s["m"]}


def _own_forward(s):
    import paper_2203_00854_amd as P
    return P.ff_gated_transition_forward(s["x"], s["w_a"], s["w_b"], s["w_o"], act=s["case"]["act"], residual=s["residual"], mask=s["mask"])


def _own_backward(s):
    import paper_2203_00854_amd as P
    dx, dw_a, dw_b, dw_o = P.ff_gated_transition_backward(s["x"], s["w_a"], s["w_b"], s["w_o"], s["dy"], act=s["case"]["act"], mask=s["mask"])
    return {"dx": dx, "dw_a": dw_a, "dw_b": dw_b, "dw_o": dw_o}


def _own_orthogonalise(s):
    import paper_2203_00854_amd as P
    return P.ff_orthogonalise(s["x"], steps=s["case"]["steps"], coefficients=COEFFICIENTS, eps=EPS)


def _own_muon(s):
    import paper_2203_00854_amd as P
    P.ff_muon_step(s["plan"], nesterov=s["case"]["nesterov"], steps=5, coefficients=COEFFICIENTS, eps=EPS, scale=s["case"]["scale"], **HYPER)
    return {"p": s["p"], "master": s["master"], "m": s["m"]}


_run_plain = {"forward": _plain_forward, "backward": _plain_backward, "orthogonalise": _plain_orthogonalise, "muon": _plain_muon}
_run_own = {"forward": _own_forward, "backward": _own_backward, "orthogonalise": _own_orthogonalise, "muon": _own_muon}


# --------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalise":
        return _polar64(s["x"].double(), case["steps"])
    if case["op"] == "muon":
        return _muon64(s)
    rows = case["rows"]
    w_a, w_b, w_o = s["w_a"].double(), s["w_b"].double(), s["w_o"].double()
    part = max(1, min(rows, (1 << 28) // max(case["c"], case["f"])))            # rows at a time: hidden layers of 2 GiB
    if case["op"] == "forward":
        y = torch.empty(rows, case["c"], dtype=torch.float64, device=DEV)
        for at in range(0, rows, part):
            here = slice(at, min(rows, at + part))
            h, _ = _hidden64(case, s["x"][here].double(), w_a, w_b)
            y[here] = torch.matmul(h, w_o.mT)
            if s["mask"] is not None:
                y[here][s["mask"][here] == 0] = 0.0
            if s["residual"] is not None:
                y[here] += s["residual"][here].double()
        return y
    dx = torch.empty(rows, case["c"], dtype=torch.float64, device=DEV)
    sums = [torch.zeros_like(w) for w in (w_a, w_b, w_o)]
    for at in range(0, rows, part):
        here = slice(at, min(rows, at + part))
        x, dy = s["x"][here].double(), s["dy"][here].double()
        if s["mask"] is not None:
            gone = s["mask"][here] == 0
            x[gone], dy[gone] = 0.0, 0.0
        x.requires_grad_()
        ws = [w.detach().requires_grad_() for w in (w_a, w_b, w_o)]
        with torch.enable_grad():
            h, _ = _hidden64(case, x, ws[0], ws[1])
            found = torch.autograd.grad(torch.matmul(h, ws[2].mT), [x, *ws], dy)
        dx[here] = found[0]
        for total, more in zip(sums, found[1:]):
            total += more
    return {"dx": dx, "dw_a": sums[0], "dw_b": sums[1], "dw_o": sums[2]}


def _hidden64(case, x, w_a, w_b):
    a, b = torch.matmul(x, w_a.mT), torch.matmul(x, w_b.mT)
    gate = {"silu": lambda: a * torch.sigmoid(a), "sigmoid": lambda: torch.sigmoid(a), "gelu": lambda: a * 0.5 * torch.erfc(-a * 2 ** -0.5)}[case["act"]]()
    return gate * b, gate


def _polar64(g, steps):
    """Newton-Schulz steps on the side that is shorter, without transposing: p(X X^T) X or X p(X^T X)."""
    x = g / (torch.linalg.matrix_norm(g, keepdim=True) + EPS)
    k1, k3, k5 = COEFFICIENTS
    left = x.shape[-2] <= x.shape[-1]
    for _ in range(steps):
        gram = torch.matmul(x, x.mT) if left else torch.matmul(x.mT, x)
        poly = k3 * gram + k5 * torch.linalg.matrix_power(gram, 2)
        poly.diagonal(dim1=-2, dim2=-1).add_(k1)
        x = torch.matmul(poly, x) if left else torch.matmul(x, poly)
    return x


def _muon64(s):
    case, beta = s["case"], HYPER["beta"]
    out = {"p": [], "master": [], "m": []}
    for i, g in enumerate(s["g"]):
        g = g.double()
        m = torch.lerp(g, s["m"][i].double(), beta)
        update = _polar64(torch.lerp(g, m, beta) if case["nesterov"] else m, 5)
        w = (s["master"][i] if s["master"] else s["p"][i]).double()
        rows, cols = g.shape[1:]
        size = math.sqrt(max(rows, cols) / cols) if case["scale"] == "spectral" else math.sqrt(0.04 * max(rows, cols))
        w = w * (1 - HYPER["lr"] * DECAY) - HYPER["lr"] * size * update
        out["p"].append(w)
        out["m"].append(m)
        if s["master"]:
            out["master"].append(w)
    return out


# --------------------------------------------------------------------------------------------------- what a pass cannot do without
def _products(rows, cols, steps):
    """A and A^2 are symmetric: half of each; then the polynomial times X."""
    n, m = min(rows, cols), max(rows, cols)
    return steps * (n * n * m + n ** 3 + 2 * n * n * m)


def work(case):
    if case["op"] in ("forward", "backward"):
        rows, c, f, size = case["rows"], case["c"], case["f"], 4 if case["dtype"] == "f32" else 2
        mask = 4 * rows if case["masked"] else 0
        if case["op"] == "forward":
            return {"bytes": size * (rows * c * (3 if case["residual"] else 2) + 3 * c * f) + mask, "flops": 6 * rows * c * f}
        return {"bytes": size * (3 * rows * c + 6 * c * f) + mask, "flops": 16 * rows * c * f}
    if case["op"] == "orthogonalise":
        return {"bytes": 2 * case["count"] * case["rows"] * case["cols"] * (4 if case["dtype"] == "f32" else 2),
                "flops": case["count"] * _products(case["rows"], case["cols"], case["steps"])}
    shapes = _shapes(case)
    total = sum(n * r * c for (r, c), n in shapes.items())
    weights = {"f32": 8, "bf16": 4, "master": 10}[case["param"]]        # read and written; beside a master copy p is only written
    return {"bytes": total * ((4 if case["grad"] == "f32" else 2) + 8 + weights), "flops": sum(n * _products(r, c, 5) for (r, c), n in shapes.items())}
