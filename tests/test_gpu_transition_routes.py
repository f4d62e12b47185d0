"""GPU parity of the gated transition on the ways through its kernels that few calls take: each tile size of each product with each activation, the weights' gradients by tiles of 256
behind rows in registers, several chunks of rows with them, wide tokens.

Bounds are those of the float64 oracle (oracle/transition.py).  What has too many rows for it is held in norm to float64 sums on the GPU.
"""
import numpy as np
import pytest
import torch

import paper_2203_00854_amd as P
from oracle import transition as T
from test_gpu_transition import DEV, HALF, Problem, n64

pytestmark = pytest.mark.gpu

# bfloat16: what forms the hidden layer, the output, the weights' gradients.  Tiles of 256 x 128 (or, in the backward pass, 128 x 128), 128 x 64 or 128, 64, 32 by how many there are.
ROUTES = [(9000, 256, 256),       # rows in registers, eight times 32 channels; weights' gradients by 256 x 256
          (12000, 190, 300),      # six times 32, and ends inside all tiles
          (7000, 512, 1040),      # large tiles; 128 x 128 for the output and dx
          (14000, 512, 1040),     # large tiles for all, 65 stages of k
          (2000, 512, 300),       # 64 x 64 for all
          (1500, 300, 700)]       # 64 x 64, 32 x 32 for the output and dx


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("rows,c,f", ROUTES)
def test_routes(rows, c, f, masked):
    p = Problem(rows, c, f, "bf16", masked, residual=True)
    p.check_forward(p.forward())
    p.check_backward(p.backward())


@pytest.mark.parametrize("act", ["gelu", "sigmoid"])
@pytest.mark.parametrize("rows,c,f,dtype", [(100, 32, 33, "bf16"), (4000, 96, 130, "bf16"), (1500, 190, 100, "bf16"), (2000, 250, 61, "bf16"), (9000, 256, 256, "bf16"),     # rows in registers
                                            (300, 300, 96, "bf16"), (2000, 512, 300, "bf16"), (3000, 272, 544, "bf16"), (7000, 320, 1040, "bf16"),                     # tiles, least to large
                                            (2000, 512, 300, "f32")])
def test_activations(rows, c, f, dtype, act):
    p = Problem(rows, c, f, dtype, masked=True)
    for w in p.w[:2]:
        w *= 3                                  # into the activations' tails
    p.check_forward(p.forward(act), act)
    p.check_backward(p.backward(act), act)


def weights_gradients(p, act="silu", part=1 << 17):
    """Those of the weights, in float64 on the GPU."""
    w_a, w_b, w_o = (w.double() for w in p.w)
    out = [torch.zeros_like(w) for w in (w_a, w_b, w_o)]
    for at in range(0, p.x.shape[0], part):
        x, dy = p.x[at:at + part].double(), p.dy[at:at + part].double()
        if p.mask is not None:
            gone = p.mask[at:at + part] == 0
            x[gone], dy[gone] = 0.0, 0.0
        a, b = x @ w_a.T.contiguous(), x @ w_b.T.contiguous()
        s = torch.sigmoid(a)
        dh = dy @ w_o
        for t, (left, right) in zip(out, ((dh * b * (s * (1 + a * (1 - s))), x), (dh * (a * s), x), (dy, a * s * b))):
            t += left.T.contiguous() @ right
    return out


def check_weights(p, dw):
    """Sums over rows, of terms of any sign.  h, da and db are off by half a step at most (bfloat16), each by one of its own, so a sum of them by no more than that of its size in norm; float32 sums
    of n terms by 2^-24 (n / 2)^(1/2), eight deviations; a, b, dh and the activation by 64 units."""
    rows = p.x.shape[0]
    for name, got, want in zip(("dw_a", "dw_b", "dw_o"), dw, weights_gradients(p)):
        off = (got.double() - want).norm() / want.norm()
        bound = (HALF[p.x.dtype] if p.x.dtype == torch.bfloat16 else 0.0) + (8 * rows ** 0.5 + 64) * T.U
        print(f"{name}: {off:.2e} of {bound:.2e}", flush=True)
        assert off <= bound, name


@pytest.mark.parametrize("masked", [False, True])
def test_rows_in_registers_in_two_chunks(masked):
    """A chunk of 1024 hidden channels in bfloat16 is 262144 rows; the second one has 300, which leave most parts of its sums over rows empty."""
    rows, c, f = (1 << 18) + 300, 32, 1024
    room = [P.ff_gated_transition_backward_workspace_bytes(P.TransitionDesc(P.FF_BF16, P.FF_SILU, c, f, n)) for n in (1 << 18, rows)]
    assert room[0] == room[1]
    p = Problem(rows, c, f, "bf16", masked)
    dx, *dw = p.backward(grad_dtype=torch.float32)
    check_weights(p, dw)
    for part in (slice(0, 200), slice((1 << 18) - 100, (1 << 18) + 100), slice(rows - 200, rows)):
        q = Problem(200, c, f, "bf16")
        q.w, q.x, q.dy, q.mask = p.w, p.x[part], p.dy[part], p.mask[part] if masked else None
        args = n64(q.x), *map(n64, q.w), n64(q.dy), "silu"
        off = np.abs(n64(dx[part]) - T.backward(*args, mask=n64(q.mask))[0])
        assert np.all(off <= T.backward_bound(*args, HALF[q.x.dtype], HALF[q.x.dtype], mask=n64(q.mask))[0]), part


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_of_wide_tokens(dtype):
    p = Problem(40000, 8192, 1, dtype)
    check_weights(p, p.backward(grad_dtype=torch.float32)[1:])
    y = p.forward()
    for part in (slice(0, 40), slice(39960, 40000)):
        q = Problem(40, 8192, 1, dtype)
        q.w, q.x = p.w, p.x[part]
        q.check_forward(y[part])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_channels(dtype):
    """8192 channels with 32768 hidden ones, weights of up to 1 GiB; unaligned tensors are copied."""
    for gap in (0, 1):
        p = Problem(3, 8192, 32768, dtype, gap=gap)
        dx, *dw = p.backward(grad_dtype=torch.float32)
        check_weights(p, dw)
        del dw
        w_a, w_b, w_o = (w.double() for w in p.w)
        x, dy = p.x.double(), p.dy.double()
        a, b, dh = x @ w_a.T, x @ w_b.T, dy @ w_o
        s = torch.sigmoid(a)
        want = (a * s * b) @ w_o.T, (dh * b * (s * (1 + a * (1 - s)))) @ w_a + (dh * (a * s)) @ w_b
        # as in check_weights, for sums of 32768 terms behind sums of 8192, and the results' own rounding
        bound = (8 * 32768 ** 0.5 + 64) * T.U + (2 * HALF[p.x.dtype] if dtype == "bf16" else 0.0)
        for name, got, exact in zip(("y", "dx"), (p.forward(), dx), want):
            off = (got.double() - exact).norm() / exact.norm()
            print(f"{name} {dtype} gap {gap}: {off:.2e} of {bound:.2e}", flush=True)
            assert off <= bound, name
        del w_a, w_b, w_o
