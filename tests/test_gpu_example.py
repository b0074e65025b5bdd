"""examples/residual_blocks.py: norms, convolutions, dropout and joins together, a training step's gradients against 64 bits, and training."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import norm_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_blocks", os.path.join(ROOT, "examples", "residual_blocks.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("blocks, N, C, H, p", [(1, 2, 8, 9, 0.0), (2, 3, 17, 13, 0.3), (3, 2, 24, 14, 0.1)])
def test_gradients_of_a_step(example, blocks, N, C, H, p):
    """torch's float64 autograd on the CPU, with the masks of norm_reference.py.  The convolutions are held to 1e-4 of their largest output by
    their own tests and measure below 2e-6; through `blocks` of them and their gradients, with rstd near one and some ten times that allowed for the
    sums between: 1e-4 of each gradient's largest value."""
    net = example.Blocks(blocks, N, C, H, p=p, seed=5)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(9)
        x, dy = (torch.randn(net.shape, generator=g, device="cuda") for _ in range(2))
        for v in net.gamma + net.beta:
            v.add_(torch.randn(v.shape, generator=g, device="cuda"), alpha=0.3)
        step = 4
        y = net.forward(x, step).clone()
        dx = net.backward(dy, step)
        leaf = lambda t: t.double().cpu().requires_grad_()  # noqa: E731
        x64, w, gamma, beta = leaf(x), [leaf(t) for t in net.w], [leaf(t) for t in net.gamma], [leaf(t) for t in net.beta]

        def norm(z, k):
            mean, var = z.mean(1, keepdim=True), z.var(1, unbiased=False, keepdim=True)
            return (z - mean) / torch.sqrt(var + example.EPS) * gamma[k].view(1, -1, 1, 1) + beta[k].view(1, -1, 1, 1)

        z, out = x64, norm(x64, 0)
        for l in range(blocks):
            drop = net.drop(step, l)
            keep = ref.kept((N, C, H, H), p, drop.seed, drop.sequence) * float(ref.scale(p))
            z = z + torch.nn.functional.conv2d(out, w[l], padding=3) * torch.from_numpy(keep)
            out = norm(z, l + 1)
        out.backward(dy.double().cpu())
        pairs = [(y, out.detach()), (dx, x64.grad)] + [(a, b.grad) for a, b in zip(net.dw + net.dgamma + net.dbeta, w + gamma + beta)]
        for got, want in pairs:
            off = float((got.double().cpu() - want).abs().max() / want.abs().max())
            assert off < 1e-4, off
    finally:
        net.close()


def test_it_learns(example):
    """The error falls to less than half, and the same seeds give the same steps again."""
    runs = []
    for _ in range(2):
        net = example.Blocks(2, 4, 16, 16, p=0.1, seed=1)
        try:
            g = torch.Generator(device="cuda")
            g.manual_seed(3)
            x = torch.randn(net.shape, generator=g, device="cuda")
            target = torch.nn.functional.avg_pool2d(x, 5, 1, 2) * 5
            runs.append(example.train(net, x, target, 40, 2.0))
        finally:
            net.close()
    assert np.array_equal(runs[0], runs[1])
    assert runs[0][-1] < 0.5 * runs[0][0], runs[0]
