"""Trains one MoE layer with the library: routing and the exact quantile bias, the experts'
rows, the balance loss with the router backward, AdamW.

    python examples/train_moe.py [--steps 60] [--balance eqb|loss|both|none] [--state-bits 8|32]

The layer y_t = sum over the chosen experts of sigmoid(z_te) FFN_e(x_t), z = x W_r, learns a
random teacher on synthetic inputs whose clusters load the experts unevenly.  The experts'
products are the program's own (torch matrix products over each expert's rows); everything
around them are calls of the library.  Prints the error, the balance loss and MaxVio.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_28053_amd import eqb  # noqa: E402
from paper_2609_28053_amd.train import AdamW, BalanceLoss, ExpertRows  # noqa: E402


class MoeLayer:
    def __init__(self, T, E, K, H, F, P, alpha, state_bits, lr, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        new = lambda *s, scale: torch.randn(s, generator=g, device=device) * scale  # noqa: E731
        self.T, self.E, self.K, self.P = T, E, K, P
        self.router = new(H, E, scale=H ** -0.5)
        self.up, self.down = new(E, H, F, scale=H ** -0.5), new(E, F, H, scale=F ** -0.5)
        self.bias = torch.zeros(E, device=device)
        # the weights that the products use: BF16 copies that the optimizer keeps
        params = [self.router, self.up, self.down]
        self.copies = [p.to(torch.bfloat16) for p in params]
        self.opt = AdamW(params, lr=lr, weight_decay=[0.0, 0.01, 0.01], state_bits=state_bits, copies=self.copies)
        self.route = eqb.Layer(T, E, K, P, device=device)
        self.rows = ExpertRows(T, E, K, device=device)
        self.balance = BalanceLoss(T, E, K, P, alpha=alpha, device=device)
        self.part = eqb.PartOffsets([T * p // P for p in range(P + 1)])
        self.inj = torch.empty((P, E), device=device)
        self.maxvio = torch.empty(1, dtype=torch.float64, device=device)

    def forward(self, x):
        router, up, down = self.copies
        z = (x @ router).view(torch.int16)
        lay = self.route.step(z, self.bias, self.part)
        rows = self.rows.plan(lay.topk_idx).dispatch(x)
        first = self.rows.offsets.tolist()
        hidden = torch.empty((rows.shape[0], up.shape[2]), dtype=rows.dtype, device=rows.device)
        out = torch.empty_like(rows)
        for e in range(self.E):
            mine = slice(first[e], first[e + 1])
            torch.matmul(rows[mine], up[e], out=hidden[mine])
            hidden[mine].relu_()
            torch.matmul(hidden[mine], down[e], out=out[mine])
        y = self.rows.combine(out, lay.topk_score)
        loss = self.balance.forward(z, load=lay.load_out, part_off=self.part)
        eqb.eqb_max_violation(lay.load_out, self.T, self.K, self.maxvio, part_off=self.part)
        return y, loss, (x, z, rows, hidden, out, first)

    def backward(self, grad_y, saved, use_loss, eta):
        x, z, rows, hidden, out, first = saved
        router, up, down = self.copies
        lay = self.route
        grad_out, grad_score = self.rows.combine_backward(grad_y, out, lay.topk_score)
        grad_up, grad_down = torch.empty_like(self.up), torch.empty_like(self.down)
        grad_rows = torch.empty_like(rows)
        for e in range(self.E):
            mine = slice(first[e], first[e + 1])
            grad_down[e] = hidden[mine].t() @ grad_out[mine]
            grad_h = (grad_out[mine] @ down[e].t()) * (hidden[mine] > 0)
            grad_up[e] = rows[mine].t() @ grad_h
            grad_rows[mine] = grad_h @ up[e].t()
        grad_x = self.rows.combine(grad_rows)
        inj = None
        if eta:
            eqb.eqb_lei_residual(lay.load_out, self.T, self.K, eta, 1.0, self.inj, self.part)
            inj = self.inj
        grad_loss = torch.full((self.P,), (1.0 / self.P) if use_loss else 0.0, device=x.device)
        grad_z = self.balance.backward(z, grad_loss, topk_idx=lay.topk_idx, grad_score=grad_score, inj=inj,
                                       part_off=self.part)
        grad_x = grad_x + (grad_z.to(torch.bfloat16) @ router.t())       # what a layer below would take
        return [x.t().to(torch.float32) @ grad_z, grad_up, grad_down], grad_x


def train(steps=60, balance="eqb", state_bits=8, T=4096, E=16, K=2, H=64, F=96, P=4, lr=3e-3, alpha=1e-2, eta=0.0,
          seed=0, say=print):
    """Returns the history of (mean square error, mean balance loss, MaxVio)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    layer = MoeLayer(T, E, K, H, F, P, alpha, state_bits, lr, seed)
    centres = torch.randn((24, H), generator=g, device="cuda") * 1.5
    share = torch.arange(1, 25, device="cuda", dtype=torch.float32) ** -1.0
    teacher = torch.randn((H, H), generator=g, device="cuda") * H ** -0.5
    history = []
    for step in range(steps):
        which = torch.multinomial(share, T, replacement=True, generator=g)
        x = (centres[which] + torch.randn((T, H), generator=g, device="cuda")).to(torch.bfloat16)
        target = torch.tanh(x.to(torch.float32) @ teacher)
        y, loss, saved = layer.forward(x)
        error = y.to(torch.float32) - target
        grads, _ = layer.backward((error * (2.0 / T)).to(torch.bfloat16), saved, balance in ("loss", "both"), eta)
        layer.opt.step(grads)
        if balance in ("eqb", "both"):
            layer.bias.copy_(layer.route.b_next)
        history.append((float(error.square().mean()), float(loss.mean()), float(layer.maxvio)))
        if step % 10 == 0 or step == steps - 1:
            say("step %3d  error %.4f  balance loss %.5f  MaxVio %.3f" % (step, *history[-1]))
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--balance", choices=("eqb", "loss", "both", "none"), default="eqb")
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--alpha", type=float, default=1e-2, help="weight of the balance loss")
    ap.add_argument("--eta", type=float, default=0.0, help="load-error injection")
    a = ap.parse_args()
    train(a.steps, a.balance, a.state_bits, alpha=a.alpha, eta=a.eta)


if __name__ == "__main__":
    main()
