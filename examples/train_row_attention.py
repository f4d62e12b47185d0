"""Training of one MSA row attention module with pair bias: the library's training operators together.

    python examples/train_row_attention.py [--steps 200] [--bits 8]

The module learns to give what another one, drawn at random, gives on synthetic representations (no data is needed).  One step:

    ff_layernorm_forward of the MSA and of the pair representation, statistics kept
    projections and the attention core in plain torch (the fused modules keep nothing for a gradient)
    ff_attention_core_backward, the projections' gradients as torch products
    ff_layernorm_backward of both, the residual path's gradient added in the same pass
    ff_grad_norm, ff_adamw_step: all tensors at once, bfloat16 weights beside float32 master copies, states in 8 or 32 bits

At the end the trained weights run in the fused module, ff_gated_attention_residual.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2203_00854_amd as P  # noqa: E402

EPS = 1e-5
BF16 = torch.bfloat16


class RowAttention:
    """Weights of one module (the names of ff_attn_weights) and its gradients, kept in buffers of their own."""

    def __init__(self, c, c_z, heads, head_dim, seed, bits=8, device="cuda:0"):
        gen = torch.Generator(device).manual_seed(seed)
        hd = heads * head_dim
        draw = lambda *s: torch.randn(*s, generator=gen, device=device) / s[-1] ** 0.5  # noqa: E731
        one, zero = (lambda n: torch.ones(n, device=device)), (lambda n: torch.zeros(n, device=device))
        master = {"ln_g": one(c), "ln_b": zero(c), "lnz_g": one(c_z), "lnz_b": zero(c_z), "w_q": draw(hd, c), "w_k": draw(hd, c), "w_v": draw(hd, c),
                  "w_b": draw(heads, c_z), "w_g": draw(hd, c), "b_g": one(hd), "w_o": draw(c, hd), "b_o": zero(c)}
        self.c, self.c_z, self.heads, self.d = c, c_z, heads, head_dim
        self.names = list(master)
        self.master = master
        self.w = {k: v.to(BF16) for k, v in master.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in master.items()}
        self.plan = P.make_adamw_plan(self.w.values(), self.grad.values(), master=self.master.values(), weight_decay=[0.01 if v.dim() > 1 else 0.0 for v in master.values()],
                                      **P.adamw_states(list(self.w.values()), bits))
        self.step_no = 0

    def _heads(self, t):
        """[rows, L, H d] -> [rows, H, L, d]"""
        return t.view(t.shape[0], t.shape[1], self.heads, self.d).transpose(1, 2).contiguous()

    def _tokens(self, t):
        return t.transpose(1, 2).reshape(t.shape[0], t.shape[2], -1)

    def forward(self, m, z, mask):
        """m + module(m, z), and what the gradient needs."""
        w, (rows, length, _) = self.w, m.shape
        mn, _, m_mean, m_rstd = P.ff_layernorm_forward(m, w["ln_g"], w["ln_b"], eps=EPS)
        zn, _, z_mean, z_rstd = P.ff_layernorm_forward(z, w["lnz_g"], w["lnz_b"], eps=EPS)
        flat = mn.view(-1, self.c)
        project = lambda k: (flat @ w[k].t()).view(rows, length, -1)  # noqa: E731
        q, k, v = (self._heads(project(n)) for n in ("w_q", "w_k", "w_v"))
        g = self._heads(torch.sigmoid(project("w_g").float() + w["b_g"].float()).to(BF16))
        bias = (zn.view(-1, self.c_z) @ w["w_b"].t()).float().t().reshape(self.heads, length, length).contiguous()
        scores = torch.matmul(q.float(), k.float().transpose(2, 3).contiguous()) * self.d ** -0.5 + bias
        live = mask[:, None, None, :] != 0
        scores = scores.masked_fill(~live, float("-inf"))
        top = scores.amax(-1, keepdim=True)
        e = torch.where(live, torch.exp(scores - torch.where(top.isfinite(), top, 0.0)), 0.0)
        p = e / e.sum(-1, keepdim=True).clamp_min(1e-30)               # a row without live keys: no weight anywhere
        o = self._tokens((g.float() * torch.matmul(p, v.float())).to(BF16)).reshape(-1, q.shape[1] * self.d)
        out = (m.float() + (o @ w["w_o"].t()).float().view_as(m) + w["b_o"].float()).to(BF16)
        return out, (m, z, mask, mn, zn, m_mean, m_rstd, z_mean, z_rstd, q, k, v, g, bias, o)

    def backward(self, kept, dout):
        """Gradients of the weights into self.grad; returns (dm, dz)."""
        m, z, mask, mn, zn, m_mean, m_rstd, z_mean, z_rstd, q, k, v, g, bias, o = kept
        w, grad, (rows, length, c) = self.w, self.grad, m.shape
        into = lambda name, value: grad[name].copy_(value)  # noqa: E731
        d = dout.view(-1, c)
        into("w_o", d.t() @ o)
        into("b_o", d.float().sum(0))
        do = self._heads((d @ w["w_o"]).view(rows, length, -1))
        desc = P.CoreDesc(P.FF_BF16, rows, self.heads, length, self.d)
        dq, dk, dv, dg, dbias = P.ff_attention_core_backward(desc, q, k, v, g, bias, mask, do)
        dg = dg.float() * g.float() * (1 - g.float())
        flat = mn.view(-1, c)
        dmn = torch.zeros(flat.shape, device=m.device)
        for name, t in (("w_q", dq), ("w_k", dk), ("w_v", dv), ("w_g", dg.to(BF16))):
            t = self._tokens(t).reshape(rows * length, -1)
            into(name, t.t() @ flat)
            dmn += t @ w[name]
        into("b_g", self._tokens(dg).reshape(rows * length, -1).sum(0))
        db = dbias.view(self.heads, -1).t().to(BF16).contiguous()
        into("w_b", db.t() @ zn.view(-1, self.c_z))
        dzn = (db @ w["w_b"]).view_as(z)
        dm, _, _ = P.ff_layernorm_backward(m, w["ln_g"], dmn.to(BF16).view_as(m), mean=m_mean, rstd=m_rstd, dsum=dout, eps=EPS, dgamma=grad["ln_g"], dbeta=grad["ln_b"])
        dz, _, _ = P.ff_layernorm_backward(z, w["lnz_g"], dzn, mean=z_mean, rstd=z_rstd, eps=EPS, dgamma=grad["lnz_g"], dbeta=grad["lnz_b"])
        return dm, dz

    def update(self, lr, max_norm=0.1):
        self.step_no += 1
        norm = P.ff_grad_norm(self.plan)
        P.ff_adamw_step(self.plan, self.step_no, lr, betas=(0.9, 0.99), eps=1e-8, norm=norm, max_norm=max_norm, seed=self.step_no)
        return norm

    def fused(self, m, z, mask):
        """The same by the fused module."""
        desc = P.make_desc(P.FF_MSA_ROW, m, self.heads, self.d, self.c_z, EPS)
        return P.ff_gated_attention_residual(desc, self.w, m, z, mask)


def train(steps=200, bits=8, rows=16, length=48, c=64, c_z=32, heads=4, head_dim=16, lr=3e-3, seed=0, tell=None, device="cuda:0"):
    """Losses of the steps, and the mean square of what the trained module, run fused, is away from its teacher."""
    teacher = RowAttention(c, c_z, heads, head_dim, seed + 1, 32, device)
    student = RowAttention(c, c_z, heads, head_dim, seed + 2, bits, device)
    gen = torch.Generator(device).manual_seed(seed)

    def batch():
        m = torch.randn(rows, length, c, generator=gen, device=device).to(BF16)
        z = torch.randn(length, length, c_z, generator=gen, device=device).to(BF16)
        mask = (torch.rand(rows, length, generator=gen, device=device) < 0.9).float()
        return m, z, mask, teacher.fused(m, z, mask)

    losses = []
    for step in range(steps):
        m, z, mask, want = batch()
        out, kept = student.forward(m, z, mask)
        off = out.float() - want.float()
        losses.append(off.square().mean())
        student.backward(kept, (2 * off / off.numel()).to(BF16))
        norm = student.update(lr)
        if tell and step % 20 == 0:
            tell(f"step {step}: loss {losses[-1].item():.5f}, gradient norm {norm.item():.5f}")
    m, z, mask, want = batch()
    last = (student.fused(m, z, mask).float() - want.float()).square().mean().item()
    return [x.item() for x in losses], last


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    losses, last = train(a.steps, a.bits, tell=lambda s: print(s, flush=True))
    print(f"mean square error: {losses[0]:.5f} at the first step, {last:.5f} of the trained module run fused")


if __name__ == "__main__":
    main()
