"""The training entry points: struct layouts, plans and refusals, without a launch (CPU)."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2203_00854_amd as P
from paper_2203_00854_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, Y, S, R, G, BETA, MEAN, RSTD, WS = (0x1000000 * (i + 1) for i in range(9))


def test_struct_layouts_match_the_header():
    assert C.sizeof(B.NormDesc) == 24 and C.sizeof(B.AdamWDesc) == 16 and C.sizeof(B.AdamWTensor) == 72 and C.sizeof(B.AdamWHyper) == 56
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ff.h")).read(), flags=re.S)
    for struct, name in ((B.NormDesc, "ff_norm_desc"), (B.AdamWDesc, "ff_adamw_desc"), (B.AdamWTensor, "ff_adamw_tensor"),
                         (B.AdamWHyper, "ff_adamw_hyper")):
        body = [b for b, n in re.findall(r"typedef struct\s*\{([^{}]*)\}\s*(\w+)", text) if n == name][0]
        declared = re.findall(r"([a-z_0-9]+)\s*(?=[,;])", body)
        assert declared == [f[0] for f in struct._fields_], name


def norm_desc(**kw):
    return B.NormDesc(**{**dict(dtype=P.FF_BF16, c=64, rows=10, ln_eps=1e-5), **kw})


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(c=0), dict(c=8193), dict(rows=-1), dict(rows=1 << 41), dict(ln_eps=-1.0), dict(ln_eps=float("nan"))])
def test_layernorm_descriptors(kw):
    d = norm_desc(**kw)
    assert P.lib().ff_layernorm_backward_workspace_bytes(C.byref(d)) == 0
    assert P.last_error() != ""
    assert P.lib().ff_layernorm_forward(C.byref(d), X, None, G, BETA, None, Y, None, None, None) == B.FF_EINVAL
    assert P.lib().ff_layernorm_backward(C.byref(d), X, G, None, None, Y, None, S, MEAN, RSTD, 0, WS, 1 << 40, None) == B.FF_EINVAL


def test_layernorm_forward_refusals():
    d, f = norm_desc(), P.lib().ff_layernorm_forward
    bad = [(None, None, G, BETA, None, Y, None, None), (X, None, None, BETA, None, Y, None, None), (X, None, G, None, None, Y, None, None),
           (X, None, G, BETA, None, None, None, None), (X, R, G, BETA, None, Y, None, None), (X, None, G, BETA, S, Y, None, None),
           (X, None, G, BETA, None, Y, MEAN, None), (X, None, G, BETA, None, Y, None, RSTD), (X, None, G, BETA, None, X, None, None),
           (X, None, G, BETA, None, X + 1278, None, None), (X, R, G, BETA, S, R, None, None), (X, R, G, BETA, S, S, None, None),
           (X, R, G, BETA, X + 2, Y, None, None), (X, R, G, BETA, R + 2, Y, None, None), (X + 1, None, G, BETA, None, Y, None, None),
           (X, None, G, BETA, None, Y, MEAN + 2, RSTD)]
    for args in bad:
        assert f(C.byref(d), *args, None) == B.FF_EINVAL, args
    assert f(None, X, None, G, BETA, None, Y, None, None, None) == B.FF_EINVAL
    assert f(C.byref(norm_desc(rows=0)), None, None, None, None, None, None, None, None, None) == B.FF_OK


def test_layernorm_backward_refusals():
    d, f = norm_desc(), P.lib().ff_layernorm_backward
    need = P.ff_layernorm_backward_workspace_bytes(d)
    good = dict(s=X, gamma=G, mean=MEAN, rstd=RSTD, dy=Y, dsum=None, dx=S, dgamma=R, dbeta=BETA, accumulate=0, ws=WS, n=need)
    assert need % 256 == 0
    for kw in (dict(s=None), dict(gamma=None), dict(dy=None), dict(dx=None), dict(dgamma=None), dict(dbeta=None), dict(mean=None), dict(rstd=None),
               dict(accumulate=2), dict(dx=X), dict(dx=X + 2), dict(dx=Y + 2), dict(dsum=S + 2), dict(dbeta=R + 4), dict(dgamma=R + 2),
               dict(ws=None), dict(ws=WS + 8), dict(dy=Y + 1)):
        assert f(C.byref(d), *{**good, **kw}.values(), None) == B.FF_EINVAL, kw
        assert P.last_error() != ""
    assert f(C.byref(d), *{**good, "n": need - 1}.values(), None) == B.FF_EWORKSPACE
    assert "workspace too small" in P.last_error()


def test_backward_workspace_is_a_fraction_of_the_input():
    for rows, c in ((2048 * 2048, 128), (5120 * 384, 64), (100_000, 1024)):
        assert P.ff_layernorm_backward_workspace_bytes(norm_desc(rows=rows, c=c)) <= rows * c * 2 / 8
    assert P.ff_layernorm_backward_workspace_bytes(norm_desc(rows=0)) >= 1


def tensors(*rows):
    t = np.zeros(len(rows), np.dtype(B.AdamWTensor))
    for i, r in enumerate(rows):
        for k, v in r.items():
            t[k][i] = v
    return t


GOOD = dict(p=0x10000, g=0x20000, m=0x30000, v=0x40000, numel=5000, weight_decay=0.1)


def plan_bytes(desc, t):
    return P.lib().ff_adamw_plan_bytes(C.byref(desc), t.ctypes.data)


def test_plan_covers_every_value_once():
    d = B.AdamWDesc(P.FF_F32, P.FF_BF16, 8, 4)
    sizes = [5000, 0, 1, 8192]
    t = tensors(*({**GOOD, "p": 0x100000 * (i + 1), "g": 0x10000000 + 0x100000 * i, "m": 0x20000000 + 0x100000 * i, "v": 0x30000000 + 0x100000 * i,
                   "m_exp": 0x40000000 + 0x100000 * i, "v_exp": 0x50000000 + 0x100000 * i, "numel": n} for i, n in enumerate(sizes)))
    n = plan_bytes(d, t)
    host = np.zeros(n, np.uint8)
    assert P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, host.ctypes.data, n) == B.FF_OK
    rec = host.view(np.dtype({"names": ["p", "g", "master", "m", "v", "m_exp", "v_exp", "value", "group", "n", "decay", "tag"],
                              "formats": ["<u8"] * 7 + ["<i8", "<u4", "<i4", "<f4", "<u4"]}))[1:]
    assert rec["n"].sum() == sum(sizes) and (rec["n"] > 0).all()
    assert np.array_equal(rec["value"], np.concatenate([[0], np.cumsum(rec["n"])[:-1]]))
    groups = np.cumsum([0] + [-(-s // 256) for s in sizes])
    for r in rec:
        i = int(r["p"] // 0x100000) - 1
        at = (int(r["p"]) - 0x100000 * (i + 1)) // 4
        assert at % 256 == 0 and at + r["n"] <= sizes[i]
        assert r["g"] == t["g"][i] + 2 * at and r["m"] == t["m"][i] + at and r["v"] == t["v"][i] + at
        assert r["m_exp"] == t["m_exp"][i] + at // 256 and r["v_exp"] == t["v_exp"][i] + at // 256
        assert r["group"] == groups[i] + at // 256 and r["decay"] == np.float32(0.1) and r["master"] == 0


@pytest.mark.parametrize("desc", [(2, 0, 32, 1), (0, 5, 32, 1), (0, 0, 16, 1), (0, 0, 32, -1)])
def test_plan_descriptors(desc):
    d = B.AdamWDesc(*desc)
    assert plan_bytes(d, tensors(GOOD)) == 0
    assert P.last_error() != ""


@pytest.mark.parametrize("bits,kw", [
    (32, dict(numel=-1)), (32, dict(g=0)), (32, dict(p=0)), (32, dict(m=0)), (32, dict(v=0)), (32, dict(p=0x10002)), (32, dict(g=0x20001)),
    (32, dict(m=0x30002)), (32, dict(v=0x40001)), (32, dict(m_exp=0x50000, v_exp=0x60000)), (8, dict(m_exp=0x50000)), (8, dict(v_exp=0x50000)),
    (8, dict()), (32, dict(master=0x70000)), (32, dict(weight_decay=-0.1)), (32, dict(weight_decay=np.nan)), (32, dict(weight_decay=np.inf)),
    (32, dict(numel=1 << 41)), (0, dict(g=0)),
])
def test_plan_refusals(bits, kw):
    d = B.AdamWDesc(P.FF_F32, P.FF_F32, bits, 2)
    more = dict(m_exp=0x50000, v_exp=0x60000) if bits == 8 and not kw.keys() & {"m_exp", "v_exp"} and kw else {}
    t = tensors({**GOOD, **({"m_exp": 0x50000, "v_exp": 0x60000} if bits == 8 else {})}, {**GOOD, **more, **kw})
    assert plan_bytes(d, t) == 0, kw
    assert P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, 0x1000, 240) == B.FF_EINVAL


def test_plan_needs_its_own_size():
    d, t = B.AdamWDesc(P.FF_F32, P.FF_F32, 32, 1), tensors(GOOD)
    n = plan_bytes(d, t)
    host = np.zeros(n + 8, np.uint8)
    assert P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, host.ctypes.data, n - 1) == B.FF_EWORKSPACE
    assert P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, None, n) == B.FF_EINVAL
    assert P.lib().ff_adamw_plan_bytes(C.byref(d), None) == 0
    assert P.lib().ff_adamw_plan_bytes(None, t.ctypes.data) == 0


def test_step_and_norm_refusals():
    lib = P.lib()
    d = B.AdamWDesc(P.FF_F32, P.FF_F32, 32, 1)
    n = plan_bytes(d, tensors(GOOD))
    hyper = lambda **kw: C.byref(B.AdamWHyper(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=1.0, step=1, seed=0), **kw}))  # noqa: E731
    nan = float("nan")
    step = lambda desc=d, plan=X, size=n, h=hyper(), norm=None: lib.ff_adamw_step(C.byref(desc), plan, size, h, norm, None)  # noqa: E731
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1e-8),
               dict(step=0)):
        assert step(h=hyper(**kw)) == B.FF_EINVAL, kw
    for kw in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=nan)):
        assert step(h=hyper(**kw), norm=Y) == B.FF_EINVAL, kw
    assert step(plan=None) == B.FF_EINVAL and step(plan=X + 8) == B.FF_EINVAL
    assert step(size=n - 1) == B.FF_EINVAL and step(size=0) == B.FF_EINVAL
    assert step(h=None) == B.FF_EINVAL and step(norm=Y + 2) == B.FF_EINVAL
    assert step(desc=B.AdamWDesc(P.FF_F32, P.FF_F32, 0, 1)) == B.FF_EINVAL and "gradients alone" in P.last_error()
    need = lib.ff_grad_norm_workspace_bytes()
    norm = lambda plan=X, size=n, out=Y, ws=WS, wn=need: lib.ff_grad_norm(C.byref(d), plan, size, out, ws, wn, None)  # noqa: E731
    assert norm(plan=None) == B.FF_EINVAL and norm(out=None) == B.FF_EINVAL and norm(ws=None) == B.FF_EINVAL and norm(ws=WS + 8) == B.FF_EINVAL
    assert norm(size=n + 1) == B.FF_EINVAL and norm(wn=need - 1) == B.FF_EWORKSPACE
    assert lib.ff_adamw_moments(C.byref(d), X, n, Y + 1, None, None) == B.FF_EINVAL
    assert lib.ff_adamw_moments(C.byref(d), None, n, Y, None, None) == B.FF_EINVAL
    assert lib.ff_adamw_moments(C.byref(B.AdamWDesc(0, 0, 0, 1)), X, n, Y, None, None) == B.FF_EINVAL


def test_binding_refuses_tensors_that_a_kernel_must_not_see():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        P.ff_layernorm_forward(x, torch.ones(8), torch.ones(8))                 # not on a GPU
    with pytest.raises(ValueError):
        P.ff_layernorm_backward(x, torch.ones(8), x)
    with pytest.raises(ValueError):
        P.make_grad_plan([])
    with pytest.raises(ValueError):
        P.make_grad_plan([x])
    with pytest.raises(TypeError):
        P.make_adamw_plan([x], [x], [x.to(torch.uint8)], [x.to(torch.uint8)])    # codes without exponents
    with pytest.raises(ValueError):
        P.make_adamw_plan([x], [x], [x], [x], m_exp=[x])
    with pytest.raises(ValueError):
        P.adamw_states([x], 16)


def test_layernorm_overlaps():
    d, lib = norm_desc(), P.lib()
    fwd = lambda x=X, res=None, g=G, b=BETA, s=None, y=Y, m=MEAN, r=RSTD: lib.ff_layernorm_forward(C.byref(d), x, res, g, b, s, y, m, r, None)  # noqa: E731
    for kw in (dict(y=G), dict(y=BETA - 64), dict(y=MEAN), dict(m=RSTD + 4), dict(m=X + 8), dict(r=Y), dict(m=G), dict(r=BETA), dict(res=R, s=S, m=S), dict(res=R, s=G)):
        assert fwd(**kw) == B.FF_EINVAL, kw
        assert "overlap" in P.last_error()
    need = P.ff_layernorm_backward_workspace_bytes(d)
    bwd = lambda s=X, g=G, m=MEAN, r=RSTD, dy=Y, ds=None, dx=S, dg=R, db=BETA, ws=WS: lib.ff_layernorm_backward(C.byref(d), s, g, m, r, dy, ds, dx, dg, db, 0, ws, need, None)  # noqa: E731
    for kw in (dict(dg=X), dict(db=Y + 4), dict(dg=S), dict(dg=G), dict(db=MEAN), dict(dg=WS), dict(dx=G), dict(dx=MEAN), dict(ws=X), dict(ws=S), dict(ds=S + 2), dict(ds=WS)):
        assert bwd(**kw) == B.FF_EINVAL, kw
        assert "overlap" in P.last_error() or "itself" in P.last_error()


def test_more_pieces_than_blocks_are_refused():
    d = B.AdamWDesc(P.FF_F32, P.FF_F32, 0, 1)
    t = tensors({"g": 0x10000, "numel": 2048 * ((1 << 24) - 1)})
    n = plan_bytes(d, t)
    assert n > 0
    t["numel"] += 1
    assert plan_bytes(d, t) == 0 and "pieces" in P.last_error()
    assert P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, 0x1000, n + 80) == B.FF_EUNSUPPORTED


def test_calls_refuse_what_is_no_tensor_or_number():
    import torch
    x, g = torch.zeros(4, 8), torch.ones(8)
    for args in ((1, g, g), (x, None, g), (x, g, "beta"), (x, g, g, 3)):
        with pytest.raises(TypeError):
            P.ff_layernorm_forward(*args)
    with pytest.raises(TypeError):
        P.ff_layernorm_forward(x, g, g, eps="small")
    with pytest.raises(ValueError):
        P.ff_layernorm_forward(torch.zeros(()), g, g)
    with pytest.raises(ValueError):
        P.ff_layernorm_backward(x.to("meta"), g, x)
    with pytest.raises(TypeError):
        P.calls().grad_norm(0)


@pytest.mark.parametrize("bits", [32, 8])
def test_plan_refuses_tensors_that_overlap(bits):
    """A weight listed twice would be stepped by two blocks at a time; gradients are only read."""
    d = B.AdamWDesc(P.FF_BF16, P.FF_F32, bits, 3)
    size = dict(p=2, master=4, m=bits // 8, v=bits // 8, g=4)
    kinds = [*size] + (["m_exp", "v_exp"] if bits == 8 else [])
    space = {k: 0x1000000 * (j + 1) for j, k in enumerate(kinds)}
    clean = lambda: [{**GOOD, **{k: at + 0x40000 * i for k, at in space.items()}} for i in range(3)]  # noqa: E731

    def status(rows):
        t = tensors(*rows)
        n = plan_bytes(d, t)
        return P.lib().ff_adamw_plan(C.byref(d), t.ctypes.data, np.zeros(n, np.uint8).ctypes.data, n)

    assert status(clean()) == B.FF_OK
    rows = clean()
    rows[2]["g"] = rows[0]["g"] + 8
    assert status(rows) == B.FF_OK
    for a in kinds:
        for b in kinds:
            if a == b == "g":
                continue
            length = {k: 5000 * s for k, s in size.items()}.get(b, 20)
            rows = clean()
            rows[2][a] = rows[1][b] + length - 4             # the last four bytes of another
            assert status(rows) == B.FF_EINVAL, (a, b)
            rows[2][a] = rows[1][b] + length                 # right behind it
            assert status(rows) == B.FF_OK, (a, b)


def test_layernorm_workspace_apart_from_every_input():
    """A block that ends early writes its partial sums while others still read gamma and the statistics."""
    d, lib = norm_desc(rows=1000), P.lib()
    need = P.ff_layernorm_backward_workspace_bytes(d)
    bwd = lambda ws, g=G, m=MEAN, r=RSTD: lib.ff_layernorm_backward(C.byref(d), X, g, m, r, Y, None, S, R, BETA, 0, ws, need, None)  # noqa: E731
    for kw in (dict(ws=G), dict(ws=MEAN), dict(ws=RSTD), dict(ws=WS, g=WS + need - 2), dict(ws=WS, m=WS + need - 4), dict(ws=WS, r=WS - 3996), dict(ws=WS, g=WS - 126)):
        assert bwd(**kw) == B.FF_EINVAL, kw
        assert "the workspace overlaps" in P.last_error()


def test_norm_and_workspace_overlaps():
    """Blocks write their partial sums while others still read the plan's addresses."""
    lib, d = P.lib(), B.AdamWDesc(P.FF_F32, P.FF_F32, 32, 1)
    n, need = plan_bytes(d, tensors(GOOD)), P.lib().ff_grad_norm_workspace_bytes()
    norm = lambda out=Y, ws=WS: lib.ff_grad_norm(C.byref(d), X, n, out, ws, need, None)  # noqa: E731
    for kw in (dict(out=X), dict(out=X + n - 4), dict(ws=X), dict(ws=X + 256), dict(ws=X - need + 256), dict(out=WS), dict(out=WS + need - 4)):
        assert norm(**kw) == B.FF_EINVAL, kw
        assert "overlap" in P.last_error()


def plan_of(columns):
    """A plan's record of its tensors, on the CPU."""
    import torch
    plan = B.AdamWPlan.__new__(B.AdamWPlan)
    numel = [t.numel() for t in columns["g"]]
    table = np.zeros(len(numel), np.dtype(B.AdamWTensor))
    table["numel"] = numel
    for k, ts in columns.items():
        table[k] = [t.data_ptr() for t in ts]
    plan.tensors, plan.spans = (table, {k: (ts, ts[0].dtype) for k, ts in columns.items()}), {}
    assert torch.is_tensor(columns["g"][0])
    return plan


def test_what_shares_memory_with_a_plan():
    import torch
    room = torch.zeros(4000)
    codes = torch.zeros(3000, dtype=torch.uint8)
    exps = torch.zeros(20, dtype=torch.uint8)
    g = [room[2000:2600], room[100:100], room[100:400]]
    plan = plan_of({"g": g, "m": [codes[1000:1600], codes[7:7], codes[300:600]], "m_exp": [exps[10:13], exps[0:0], exps[4:6]]})
    for lo, hi, meets in ((0, 100, False), (99, 101, True), (100, 400, True), (399, 401, True), (400, 2000, False), (1999, 2001, True), (2599, 2601, True), (2600, 4000, False),
                          (0, 4000, True), (250, 250, False)):
        assert plan.meets(("g",), room[lo:hi]) == meets, (lo, hi)
        assert not plan.meets(("m", "m_exp"), room[lo:hi])
    for lo, hi, meets in ((0, 300, False), (299, 301, True), (599, 600, True), (600, 1000, False), (1599, 1601, True), (1600, 3000, False)):
        assert plan.meets(("m", "m_exp"), codes[lo:hi]) == meets, (lo, hi)
    for lo, hi, meets in ((0, 4, False), (5, 6, True), (6, 10, False), (12, 13, True), (13, 20, False)):
        assert plan.meets(("m", "m_exp"), exps[lo:hi]) == meets, (lo, hi)
        assert not plan.meets(("v", "g"), exps[lo:hi])
    assert not plan.meets(("g",), 3)


def test_moments_overlaps():
    """Two tensors of 5000 and 3 values are four pieces, which hold 2 x 2048 + 2 values at least."""
    lib, d = P.lib(), B.AdamWDesc(P.FF_F32, P.FF_F32, 32, 2)
    second = {k: GOOD[k] + 0x1000000 for k in ("p", "g", "m", "v")}
    n, least = plan_bytes(d, tensors(GOOD, {**GOOD, **second, "numel": 3})), 4 * (2 * 2048 + 2)
    assert n == 5 * 80
    for m, v in ((Y, Y), (Y, Y + least - 4), (Y + least - 4, Y), (X, None), (None, X + n - 4), (X - least + 4, Y), (Y, X + 16)):
        assert lib.ff_adamw_moments(C.byref(d), X, n, m, v, None) == B.FF_EINVAL, (m, v)
        assert "overlap" in P.last_error()
