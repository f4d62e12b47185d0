"""The training example: its gradients against torch's in float32, and that it learns with states of either size."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_row_attention.py")


def example():
    spec = importlib.util.spec_from_file_location("train_row_attention", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def reference(module, m, z, mask):
    """The module in float32 on the CPU with torch's gradients."""
    w = {k: v.detach().float().cpu().requires_grad_() for k, v in module.w.items()}
    m, z, mask = m.float().cpu().requires_grad_(), z.float().cpu().requires_grad_(), mask.cpu()
    rows, length, c = m.shape
    norm = torch.nn.functional.layer_norm
    mn, zn = norm(m, (c,), w["ln_g"], w["ln_b"], 1e-5), norm(z, (module.c_z,), w["lnz_g"], w["lnz_b"], 1e-5)
    split = lambda t: t.view(rows, length, module.heads, module.d).transpose(1, 2)  # noqa: E731
    q, k, v, g = (split(mn @ w[n].t()) for n in ("w_q", "w_k", "w_v", "w_g"))
    g = torch.sigmoid(g + w["b_g"].view(module.heads, 1, module.d))
    bias = (zn @ w["w_b"].t()).permute(2, 0, 1)
    s = (q @ k.transpose(2, 3) * module.d ** -0.5 + bias).masked_fill(mask[:, None, None, :] == 0, float("-inf"))
    o = (g * (s.softmax(-1) @ v)).transpose(1, 2).reshape(rows, length, -1)
    return m + o @ w["w_o"].t() + w["b_o"], w, m, z


def test_gradients_of_a_step():
    E = example()
    module = E.RowAttention(64, 32, 4, 16, seed=3)
    gen = torch.Generator(DEV).manual_seed(4)
    m = torch.randn(6, 40, 64, generator=gen, device=DEV).to(torch.bfloat16)
    z = torch.randn(40, 40, 32, generator=gen, device=DEV).to(torch.bfloat16)
    mask = (torch.rand(6, 40, generator=gen, device=DEV) < 0.8).float()
    dout = torch.randn(6, 40, 64, generator=gen, device=DEV).to(torch.bfloat16)
    out, kept = module.forward(m, z, mask)
    dm, dz = module.backward(kept, dout)
    want, w, m32, z32 = reference(module, m, z, mask)
    want.backward(dout.float().cpu())
    # bfloat16 operands throughout: some ten roundings of 2^-9 (root mean square about 2^-10 each) on the way of any gradient
    for name, got, ref in [("out", out, want), ("dm", dm, m32.grad), ("dz", dz, z32.grad)] + [(k, module.grad[k], w[k].grad) for k in module.names]:
        # (lnz_b moves all logits of a query alike, so its gradient is zero: what is left of the sum is held against lnz_g's)
        size = w["lnz_g"].grad.norm() if name == "lnz_b" else ref.norm()
        off = ((got.float().cpu() - ref).norm() / size).item()
        print(f"{name}: {off:.2e}", flush=True)
        assert off < 2e-2, name


@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns(bits):
    losses, last = example().train(steps=120, bits=bits)
    print(bits, losses[0], losses[-1], last)
    assert last < 0.5 * losses[0]
