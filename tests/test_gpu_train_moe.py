"""The operators together: an MoE layer's gradients through the library's calls against
autograd in binary64, and the example's training run."""
import os
import sys

import pytest
import torch

from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_moe
    return train_moe


def test_layer_gradients(eqb, example):  # noqa: F811
    """dL/dW_r, dL/dW_up, dL/dW_down and dL/dx of L = sum(y c) + mean balance loss, against autograd in 64 bits
    on the same BF16 weights, inputs and logits, with the routing fixed.  The layer's BF16 roundings (logits excepted:
    they are given) are of the hidden rows, the experts' rows, their gradients and y's gradient: each 2^-9 relative, up
    to five in a chain, independent over at least 64 summed elements: 1% of a gradient's norm holds them."""
    T, E, K, H, F, P = 512, 8, 2, 64, 32, 2
    layer = example.MoeLayer(T, E, K, H, F, P, alpha=0.5, state_bits=32, lr=1e-3)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    c = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    say("layer gradients")
    y, loss, saved = layer.forward(x)
    grads, grad_x = layer.backward(c, saved, True, 0.0)
    idx = layer.route.topk_idx.long()
    load = layer.route.load_out.double()

    router, up, down = (p.double().requires_grad_() for p in layer.copies)
    xd = x.double().requires_grad_()
    zd = saved[1].view(torch.bfloat16).double()
    z = xd @ router
    z = z + (zd - z).detach()                          # the values that were routed, the gradient of the product
    s = torch.sigmoid(z)
    h = torch.relu(torch.einsum("th,ehf->tef", xd, up))
    o = torch.einsum("tef,efh->teh", h, down)
    yd = (s.gather(1, idx)[:, :, None] * o.gather(1, idx[:, :, None].expand(T, K, H))).sum(1)
    p = s / s.sum(1, keepdim=True)
    aux = sum(0.5 * (E * load[i] / (K * T // P) * p[i * T // P:(i + 1) * T // P].mean(0)).sum() for i in range(P)) / P
    ((yd * c.double()).sum() + aux).backward()
    yd, aux = yd.detach(), aux.detach()
    assert float((y.double() - yd).norm() / yd.norm()) < 0.01
    assert abs(float(loss.mean()) - float(aux)) < 1e-5
    for got, want in ((grads[0], router.grad), (grads[1], up.grad), (grads[2], down.grad), (grad_x, xd.grad)):
        far = float((got.double() - want).norm() / want.norm())
        say(f"relative error {far:.2e}")
        assert far < 0.01


@pytest.mark.parametrize("state_bits", [8, 32])
def test_training_run(example, state_bits):
    """The error falls by half, and the exact quantile bias brings MaxVio to a fraction of what it is without."""
    say(f"training, {state_bits}-bit states")
    with_bias = example.train(steps=60, balance="eqb", state_bits=state_bits, say=say)
    without = example.train(steps=60, balance="none", state_bits=state_bits, say=say)
    assert with_bias[-1][0] < 0.5 * with_bias[0][0]
    mean = lambda h: sum(v[2] for v in h[-10:]) / 10  # noqa: E731
    assert mean(with_bias) < 0.5 * mean(without)


def test_balance_loss_lowers_the_imbalance(example):
    """With the loss alone (a large weight) the last steps are more even than without it."""
    on = example.train(steps=80, balance="loss", alpha=1.0, lr=1e-2, say=say)
    off = example.train(steps=80, balance="none", alpha=1.0, lr=1e-2, say=say)
    mean = lambda h, i: sum(v[i] for v in h[-10:]) / 10  # noqa: E731
    assert mean(on, 1) < mean(off, 1) and mean(on, 2) < mean(off, 2)


def test_example_command():
    """The command itself, a few steps, in a child process."""
    import subprocess
    res = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "train_moe.py"), "--steps", "3", "--balance", "both",
                          "--eta", "1e-4"], capture_output=True, text=True, timeout=100, cwd=ROOT)
    assert res.returncode == 0, res.stderr[-2000:]
    assert "step   2" in res.stdout
