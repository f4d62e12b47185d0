"""The transition's and the matrix optimiser's entry points: struct layouts, plans and refusals, without a launch (CPU)."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2203_00854_amd as P
from paper_2203_00854_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, WA, WB, WO, DY, MASK, Y, DWA, DWB, DWO, WS, R = (0x10000000 * (i + 1) for i in range(12))
LOTS = 1 << 40


def test_struct_layouts_match_the_header():
    assert [C.sizeof(s) for s in (B.TransitionDesc, B.OrthogonaliseDesc, B.MuonDesc, B.MuonTensor, B.MuonHyper)] == [24, 56, 12, 48, 72]
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ff.h")).read(), flags=re.S)
    for struct, name in ((B.TransitionDesc, "ff_transition_desc"), (B.OrthogonaliseDesc, "ff_orthogonalise_desc"), (B.MuonDesc, "ff_muon_desc"),
                         (B.MuonTensor, "ff_muon_tensor"), (B.MuonHyper, "ff_muon_hyper")):
        body = [b for b, n in re.findall(r"typedef struct\s*\{([^{}]*)\}\s*(\w+)", text) if n == name][0]
        assert re.findall(r"([a-z_0-9]+)\s*(?=[,;])", body) == [f[0] for f in struct._fields_], name
    for enum, values in (("ff_act", ("FF_SILU", "FF_GELU", "FF_SIGMOID")), ("ff_muon_scale", ("FF_MUON_SPECTRAL", "FF_MUON_RMS"))):
        body = [b for b, n in re.findall(r"typedef enum\s*\{([^{}]*)\}\s*(\w+)", text) if n == enum][0]
        assert {k: int(v) for k, v in re.findall(r"(\w+) = (\d+)", body)} == {v: getattr(P, v) for v in values}


def transition(**kw):
    return B.TransitionDesc(**{**dict(dtype=P.FF_BF16, act=P.FF_SILU, c=64, f=96, rows=10), **kw})


FORWARD = dict(x=X, w_a=WA, w_b=WB, w_o=WO, residual=None, mask=None, y=Y, ws=WS, n=LOTS)
BACKWARD = dict(x=X, w_a=WA, w_b=WB, w_o=WO, dy=DY, mask=None, dx=Y, dw_a=DWA, dw_b=DWB, dw_o=DWO, grad_dtype=P.FF_BF16, accumulate=0, ws=WS, n=LOTS)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(act=3), dict(act=-1), dict(c=0), dict(c=8193), dict(f=0), dict(f=32769), dict(rows=-1), dict(rows=1 << 41), dict(rows=1 << 36)])
def test_transition_descriptors(kw):
    d = C.byref(transition(**kw))
    assert P.lib().ff_gated_transition_forward_workspace_bytes(d) == 0 and P.last_error() != ""
    assert P.lib().ff_gated_transition_backward_workspace_bytes(d) == 0
    assert P.lib().ff_gated_transition_forward(d, *FORWARD.values(), None) == B.FF_EINVAL
    assert P.lib().ff_gated_transition_backward(d, *BACKWARD.values(), None) == B.FF_EINVAL


def test_transition_forward_refusals():
    d, f = transition(), P.lib().ff_gated_transition_forward
    need = P.ff_gated_transition_forward_workspace_bytes(d)
    for kw in (dict(x=None), dict(w_a=None), dict(w_b=None), dict(w_o=None), dict(y=None), dict(x=X + 1), dict(w_o=WO + 1), dict(y=Y + 1), dict(residual=R + 1), dict(mask=MASK + 2),
               dict(y=X), dict(y=X + 1278), dict(y=WA), dict(y=WO + 100), dict(residual=Y + 2), dict(residual=Y - 1278), dict(mask=Y + 4), dict(ws=None), dict(ws=WS + 128),
               dict(ws=X), dict(ws=WB), dict(ws=Y), dict(residual=R, ws=R), dict(mask=MASK, ws=MASK)):
        assert f(C.byref(d), *{**FORWARD, **kw}.values(), None) == B.FF_EINVAL, kw
        assert P.last_error() != ""
    assert f(C.byref(d), *{**FORWARD, "n": need - 1}.values(), None) == B.FF_EWORKSPACE
    assert "workspace too small" in P.last_error()
    assert f(None, *FORWARD.values(), None) == B.FF_EINVAL
    assert f(C.byref(transition(rows=0)), *[None] * 8, 0, None) == B.FF_OK


def test_transition_backward_refusals():
    d, f = transition(), P.lib().ff_gated_transition_backward
    need = P.ff_gated_transition_backward_workspace_bytes(d)
    for kw in ([{k: None} for k in ("x", "w_a", "w_b", "w_o", "dy", "dx", "dw_a", "dw_b", "dw_o", "ws")] +
               [dict(grad_dtype=2), dict(accumulate=2), dict(x=X + 1), dict(dy=DY + 1), dict(dx=Y + 1), dict(dw_a=DWA + 1), dict(mask=MASK + 2), dict(dx=X), dict(dx=DY), dict(dx=WA),
                dict(mask=Y), dict(dw_a=WA), dict(dw_o=X), dict(dw_a=DWB + 2), dict(dw_o=Y), dict(ws=WS + 64), dict(ws=X), dict(ws=DWA), dict(mask=MASK, dw_b=MASK)]):
        assert f(C.byref(d), *{**BACKWARD, **kw}.values(), None) == B.FF_EINVAL, kw
        assert P.last_error() != ""
    assert f(C.byref(d), *{**BACKWARD, "n": need - 1}.values(), None) == B.FF_EWORKSPACE
    # float32 gradients of bfloat16 weights take twice the room
    assert f(C.byref(d), *{**BACKWARD, "grad_dtype": P.FF_F32, "dw_b": DWA + 64 * 96 * 2}.values(), None) == B.FF_EINVAL


@pytest.mark.parametrize("dtype", [P.FF_F32, P.FF_BF16])
def test_workspaces_hold_hidden_tensors_of_a_chunk_of_rows_only(dtype):
    for c, f in ((128, 512), (512, 2048), (16, 2048), (1000, 37)):
        d = transition(dtype=dtype, c=c, f=f, rows=1 << 30 if c == 16 else 1 << 27)
        forward, backward = P.ff_gated_transition_forward_workspace_bytes(d), P.ff_gated_transition_backward_workspace_bytes(d)
        # three hidden tensors and copies of x and dy of at most 512 MiB each, weights and partial sums
        assert forward <= (2 << 29) + (1 << 28) and backward <= (5 << 29) + (1 << 28)


def ortho(**kw):
    return B.OrthogonaliseDesc(**{**dict(dtype=P.FF_F32, count=3, rows=20, cols=200, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7), **kw})


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(count=-1), dict(rows=0), dict(cols=0), dict(rows=32769), dict(cols=32769), dict(steps=0), dict(steps=65), dict(a=float("nan")),
                                dict(b=float("inf")), dict(c=1e300), dict(eps=-1.0), dict(eps=float("nan")), dict(count=1 << 30, rows=1000)])
def test_orthogonalise_descriptors(kw):
    d = C.byref(ortho(**kw))
    assert P.lib().ff_orthogonalise_workspace_bytes(d) == 0 and P.last_error() != ""
    assert P.lib().ff_orthogonalise(d, X, Y, WS, LOTS, None) == B.FF_EINVAL


def test_orthogonalise_refusals():
    d, f = ortho(), P.lib().ff_orthogonalise
    need = P.ff_orthogonalise_workspace_bytes(d)
    for args in ((None, Y, WS), (X, None, WS), (X, Y, None), (X + 2, Y, WS), (X, Y + 2, WS), (X, X + 4, WS), (X + 4, X, WS), (X, Y, WS + 8), (X, Y, X), (X, Y, Y)):
        assert f(C.byref(d), *args, LOTS, None) == B.FF_EINVAL, args
    assert f(C.byref(d), X, Y, WS, need - 1, None) == B.FF_EWORKSPACE
    assert f(C.byref(ortho(count=0)), None, None, None, 0, None) == B.FF_OK


GOOD = dict(p=0x100000, g=0x2000000, m=0x4000000, rows=150, cols=200, weight_decay=0.1)


def matrices(*rows):
    t = np.zeros(len(rows), np.dtype(B.MuonTensor))
    for i, r in enumerate(rows):
        for k, v in r.items():
            t[k][i] = v
    return t


def muon(param=P.FF_F32, grad=P.FF_F32, n=1):
    return B.MuonDesc(param, grad, n)


def plan_of(desc, t):
    n = P.lib().ff_muon_plan_bytes(C.byref(desc), t.ctypes.data)
    host = np.zeros(n, np.uint8)
    assert P.lib().ff_muon_plan(C.byref(desc), t.ctypes.data, host.ctypes.data, n) == B.FF_OK
    return host


@pytest.mark.parametrize("desc,kw", [((2, 0, 1), {}), ((0, 3, 1), {}), ((0, 0, -1), {}), ((0, 0, 1), dict(rows=-1)), ((0, 0, 1), dict(cols=32769)), ((0, 0, 1), dict(p=0)), ((0, 0, 1), dict(g=0)),
                                     ((0, 0, 1), dict(m=0)), ((0, 0, 1), dict(p=0x100002)), ((0, 0, 1), dict(g=0x2000001)), ((0, 1, 1), dict(g=0x2000001)), ((0, 0, 1), dict(m=0x4000002)),
                                     ((0, 0, 1), dict(master=0x7000000)), ((1, 0, 1), dict(master=0x7000002)), ((0, 0, 1), dict(weight_decay=-0.1)), ((0, 0, 1), dict(weight_decay=np.nan))])
def test_muon_plan_refusals(desc, kw):
    d, t = B.MuonDesc(*desc), matrices({**GOOD, **kw})
    assert P.lib().ff_muon_plan_bytes(C.byref(d), t.ctypes.data) == 0 and P.last_error() != ""
    host = np.zeros(1 << 16, np.uint8)
    assert P.lib().ff_muon_plan(C.byref(d), t.ctypes.data, host.ctypes.data, host.size) == B.FF_EINVAL


def test_muon_plan_overlaps():
    size = 150 * 200 * 4
    for kw in (dict(p=0x100000), dict(p=0x100000 + size - 4), dict(m=0x4000000), dict(m=0x2000000), dict(g=0x100000), dict(p=0x4000000 + 8)):
        other = {**GOOD, "p": 0x8000000, "m": 0x9000000, **kw}
        t = matrices(GOOD, other)
        n = P.lib().ff_muon_plan_bytes(C.byref(muon(n=2)), t.ctypes.data)
        host = np.zeros(n, np.uint8)
        assert P.lib().ff_muon_plan(C.byref(muon(n=2)), t.ctypes.data, host.ctypes.data, n) == B.FF_EINVAL, kw
        assert "overlaps" in P.last_error()
    plan_of(muon(n=2), matrices(GOOD, {**GOOD, "p": 0x8000000, "m": 0x9000000}))             # gradients may share memory


def test_muon_plan_sizes():
    d, t = muon(), matrices(GOOD)
    n = P.lib().ff_muon_plan_bytes(C.byref(d), t.ctypes.data)
    host = np.zeros(n + 8, np.uint8)
    assert P.lib().ff_muon_plan(C.byref(d), t.ctypes.data, host.ctypes.data, n - 8) == B.FF_EWORKSPACE
    assert P.lib().ff_muon_plan(C.byref(d), t.ctypes.data, None, n) == B.FF_EINVAL
    assert P.lib().ff_muon_plan(C.byref(d), t.ctypes.data, host.ctypes.data + 4, n) == B.FF_EINVAL
    # no matrix at all, and matrices without values
    for t, count in ((matrices(), 0), (matrices({**GOOD, "rows": 0, "p": 0}), 1)):
        host = plan_of(muon(n=count), t)
        assert P.lib().ff_muon_workspace_bytes(C.byref(muon(n=count)), host.ctypes.data, host.size) > 0


@pytest.mark.parametrize("more", [0, 61, 62])
def test_muon_plan_has_every_place_once(more):
    """Tiles of large matrices, each once (places that are none fill up), small ones behind them in the order of their sizes; up to 64 small ones have tiles too."""
    shapes = [(64, 64), (300, 700), (128, 100), (2000, 130), (1, 5), (700, 300), (129, 1), (260, 260)] + [(20, 30)] * more
    count, small, smaller = len(shapes), *((0, 0) if 3 + more <= 64 else (1, 2 + more))
    large = count - small - smaller
    rows = [{**GOOD, "rows": r, "cols": c, "p": (3 * i + 1) << 24, "g": (3 * i + 2) << 24, "m": (3 * i + 3) << 24} for i, (r, c) in enumerate(shapes)]
    host = plan_of(muon(n=len(rows)), matrices(*rows))
    head = host[:48].view(np.dtype([("tag", "<u4"), ("matrices", "<i4"), ("batches", "<i4"), ("pieces", "<i4"), ("tris", "<i4"), ("apps", "<i4"), ("small", "<i4"), ("smaller", "<i4"),
                                    ("ws", "<i8"), ("bytes", "<i8")]))[0]
    assert (head["matrices"], head["batches"], head["small"], head["smaller"]) == (count, 1, small, smaller) and head["bytes"] == host.size
    batch = host[48:96].view(np.dtype([("ws", "<i8")] + [(n, "<i4") for n in ("piece0", "pieces", "tri0", "tris", "app0", "apps", "splits", "tri_tile", "app_tile", "beside")]))[0]
    at = 96
    found = host[at:at + 64 * count].view(np.dtype([("p", "<u8"), ("g", "<u8"), ("master", "<u8"), ("m", "<u8"), ("ws", "<i8"), ("rows", "<i4"), ("cols", "<i4"), ("piece0", "<i4"),
                                                ("pieces", "<i4"), ("decay", "<f4"), ("pad", "<i4")]))
    assert sorted((int(f["rows"]), int(f["cols"])) for f in found) == sorted(shapes)
    assert [max(int(f["rows"]), int(f["cols"])) for f in found[5:]] == [128, 64] + [30] * more + [5]
    places = host[at + 64 * count:].view("<i4").reshape(-1, 2)
    tile = lambda n, t: -(-n // t)  # noqa: E731
    pad = lambda n: -(-n // 16) * 16  # noqa: E731
    kinds = (("pieces", lambda r, c: tile(pad(r) * pad(c), 4096)), ("tris", lambda r, c: tile(pad(min(r, c)), int(batch["tri_tile"])) * (tile(pad(min(r, c)), int(batch["tri_tile"])) + 1) // 2),
             ("apps", lambda r, c: tile(pad(r), int(batch["app_tile"])) * tile(pad(c), int(batch["app_tile"]))))
    first = 0
    for kind, tiles in kinds:
        got = places[first:first + head[kind]]
        got = [tuple(g) for g in got.tolist() if g[0] >= 0]
        assert sorted(got) == [(i, k) for i in range(large) for k in range(tiles(int(found[i]["rows"]), int(found[i]["cols"])))], kind
        first += head[kind]
    spans = sorted((int(f["ws"]), int(f["ws"]) + 4 * (2 * pad(int(f["rows"])) * pad(int(f["cols"])) + 2 * pad(min(int(f["rows"]), int(f["cols"]))) ** 2)) for f in found[:large])
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and spans[-1][1] <= head["ws"]


def test_muon_step_refusals():
    d, t = muon(), matrices(GOOD)
    host = plan_of(d, t)
    need = P.lib().ff_muon_workspace_bytes(C.byref(d), host.ctypes.data, host.size)
    assert need > 0
    good = dict(lr=0.1, beta=0.9, max_norm=0.0, a=3.4, b=-4.7, c=2.0, eps=1e-7, steps=5, nesterov=1, scale=0)
    plan, ws = 0x50000000, 0x60000000
    step = lambda d=d, host=host.ctypes.data, plan=plan, n=host.size, h=good, norm=None, ws=ws, k=need: P.lib().ff_muon_step(  # noqa: E731
        None if d is None else C.byref(d), host, plan, n, None if h is None else C.byref(B.MuonHyper(**h)), norm, ws, k, None)
    for kw in (dict(d=None), dict(d=muon(param=1)), dict(d=muon(grad=1)), dict(host=None), dict(plan=None), dict(plan=plan + 8), dict(n=host.size - 16), dict(n=8), dict(h=None),
               *(dict(h={**good, **x}) for x in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta=1.0), dict(beta=-0.1), dict(eps=-1.0), dict(a=float("inf")), dict(steps=0), dict(steps=65),
                                                 dict(nesterov=2), dict(scale=2))),
               dict(norm=0x70000000), dict(norm=0x70000002, h={**good, "max_norm": 1.0}), dict(norm=ws + 4, h={**good, "max_norm": 1.0}), dict(ws=None), dict(ws=ws + 128), dict(ws=plan)):
        assert step(**kw) == B.FF_EINVAL, kw
        assert P.last_error() != ""
    assert step(k=need - 1) == B.FF_EWORKSPACE
    assert P.lib().ff_muon_workspace_bytes(C.byref(muon(grad=1)), host.ctypes.data, host.size) == 0


def test_python_entry_points_refuse_on_the_host():
    """What is found out before a GPU is needed."""
    import torch
    x, w = torch.zeros(3, 4), torch.zeros(5, 4)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.ff_gated_transition_forward(x, w, w, w.t().contiguous())
    with pytest.raises(ValueError, match="act is one of"):
        P.ff_gated_transition_forward(x, w, w, w, act="relu")
    with pytest.raises(TypeError, match="w_o is missing"):
        P.ff_gated_transition_forward(x, w, w, None)
    with pytest.raises(TypeError, match="grad_dtype"):
        P.ff_gated_transition_backward(x, w, w, w, x, grad_dtype=torch.float16)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.ff_orthogonalise(x)
    with pytest.raises(ValueError, match="a plan needs a tensor"):
        P.make_muon_plan([], [], [])
    with pytest.raises(ValueError, match="it is no matrix"):
        P.make_muon_plan([x[0]], [x[0]], [x[0]])
    with pytest.raises(ValueError, match="tensors of g"):
        P.make_muon_plan([x], [x, x], [x])
    with pytest.raises(TypeError, match="m is"):
        P.make_muon_plan([x], [x], [x.double()])
    with pytest.raises(ValueError, match="g has shape"):
        P.make_muon_plan([x], [w], [x])
    with pytest.raises(ValueError, match="not on a GPU"):
        P.make_muon_plan([x], [x], [x])
    assert [t.shape for t in P.muon_states(p for p in (x, w))["m"]] == [(3, 4), (5, 4)]
