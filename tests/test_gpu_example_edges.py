"""examples/residual_blocks.py without a single block: the first norm alone, its gradients against 64 bits."""
import numpy as np
import pytest
import torch

import norm_reference as ref
from test_gpu_example import example  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def test_no_blocks(example):  # noqa: F811
    N, C, H = 2, 24, 9
    net = example.Blocks(0, N, C, H, p=0.2, seed=5)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(9)
        x, dy = (torch.randn(net.shape, generator=g, device="cuda") for _ in range(2))
        net.dz.fill_(float("nan"))  # nothing reaches the stream from elsewhere
        net.forward(x, 0)
        dx = net.backward(dy, 0)
        z, dy64 = (t.double().cpu().numpy().reshape(N, C, H * H) for t in (x, dy))
        m, r = net.mean[0].double().cpu().numpy(), net.rstd[0].double().cpu().numpy()
        want = ref.norm_backward(dy64, z, np.ones(C), m, r)
        allowed = ref.tolerances_backward(dy64, z, np.ones(C), m, r, np.zeros_like(z), want[0], "f32", "f32", want[1], want[2])
        for got, w, t in zip((dx.reshape(N, C, H * H), net.dgamma[0], net.dbeta[0]), want, allowed):
            assert (np.abs(got.double().cpu().numpy() - w) <= t).all()
    finally:
        net.close()
