"""A few residual blocks of 7x7 convolutions in training, every step of them in the library's kernels: channels-first layer norms, the
convolutions with both gradients, dropout on each branch, and the joins with the residual stream.

    z_0 = x,  y_0 = norm(x);   for every block:  h = conv(y_l, w_l),  z_{l+1} = z_l + dropout(h),  y_{l+1} = norm(z_{l+1})

The last y is fitted to a target by gradient descent on w, gamma and beta.  Masks are drawn from (seed, step, block) and never stored.

    python examples/residual_blocks.py [--steps 20] [--blocks 2] [--batch 8] [--channels 32] [--size 28] [--dropout 0.1]
"""
import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2002_00552_amd as dwm  # noqa: E402

EPS = 1e-6


def _f32(*shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda")


def _buffer(nbytes):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Conv:
    """A same-padded convolution with its gradients: three plans, their workspaces, the transformed filters."""

    def __init__(self, N, C, H, kernel):
        shape = (N, C, H, H, C, kernel, kernel, 1, kernel // 2)
        self.fwd, self.bwd, self.wgrad = dwm.dwm_plan_create(*shape), dwm.dwm_bwd_data_plan_create(*shape), dwm.dwm_bwd_filter_plan_create(*shape)
        self.U, self.Ub = _buffer(dwm.dwm_plan_filter_bytes(self.fwd)), _buffer(dwm.dwm_bwd_data_filter_bytes(self.bwd))
        self.ws = [_buffer(n) for n in (dwm.dwm_plan_workspace_bytes(self.fwd), dwm.dwm_bwd_data_workspace_bytes(self.bwd),
                                        dwm.dwm_bwd_filter_workspace_bytes(self.wgrad))]
        for set_workspace, plan, ws in zip((dwm.dwm_plan_set_workspace, dwm.dwm_bwd_data_set_workspace, dwm.dwm_bwd_filter_set_workspace),
                                           (self.fwd, self.bwd, self.wgrad), self.ws):
            set_workspace(plan, ws.data_ptr(), ws.numel())

    def forward(self, x, w, y):
        dwm.dwm_filter_transform(self.fwd, w.data_ptr(), self.U.data_ptr(), _stream())
        dwm.dwm_conv_forward(self.fwd, x.data_ptr(), self.U.data_ptr(), y.data_ptr(), _stream())

    def backward(self, x, w, dy, dx, dw):
        dwm.dwm_bwd_data_filter_transform(self.bwd, w.data_ptr(), self.Ub.data_ptr(), _stream())
        dwm.dwm_conv_backward_data(self.bwd, dy.data_ptr(), self.Ub.data_ptr(), dx.data_ptr(), _stream())
        dwm.dwm_conv_backward_filter(self.wgrad, x.data_ptr(), dy.data_ptr(), dw.data_ptr(), _stream())

    def close(self):
        dwm.dwm_plan_destroy(self.fwd)
        dwm.dwm_bwd_data_plan_destroy(self.bwd)
        dwm.dwm_bwd_filter_plan_destroy(self.wgrad)


class Blocks:
    """`blocks` residual blocks on [N][C][H][H] maps: parameters, activations and gradients of one training step."""

    def __init__(self, blocks, N, C, H, kernel=7, p=0.1, seed=0):
        self.shape, self.blocks, self.p, self.seed = (N, C, H, H), blocks, p, seed
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.w = [torch.randn((C, C, kernel, kernel), generator=g, device="cuda") * math.sqrt(1.0 / (C * kernel * kernel)) for _ in range(blocks)]
        self.gamma = [torch.ones(C, device="cuda") for _ in range(blocks + 1)]
        self.beta = [torch.zeros(C, device="cuda") for _ in range(blocks + 1)]
        self.z = [None] + [_f32(*self.shape) for _ in range(blocks)]
        self.y = [_f32(*self.shape) for _ in range(blocks + 1)]
        self.h = _f32(*self.shape)
        self.mean, self.rstd = ([_f32(N, H * H) for _ in range(blocks + 1)] for _ in range(2))
        self.dw = [torch.empty_like(w) for w in self.w]
        self.dgamma, self.dbeta = ([_f32(C) for _ in range(blocks + 1)] for _ in range(2))
        self.dy, self.dh, self.dz, self.dx = (_f32(*self.shape) for _ in range(4))
        self.conv = Conv(N, C, H, kernel)
        self.norm = dwm.dwm_norm_plan_create(N, C, H * H, dwm.DWM_F32, dwm.DWM_F32, EPS)
        self.ws = _buffer(dwm.dwm_norm_workspace_bytes(self.norm))
        dwm.dwm_norm_set_workspace(self.norm, self.ws.data_ptr(), self.ws.numel())

    def drop(self, step, block):
        return dwm.dwm_dropout_t(self.p, self.seed, step * self.blocks + block, None)

    def forward(self, x, step):
        self.z[0] = x
        dwm.dwm_norm_forward(self.norm, x.data_ptr(), self.gamma[0].data_ptr(), self.beta[0].data_ptr(), self.y[0].data_ptr(),
                             self.mean[0].data_ptr(), self.rstd[0].data_ptr(), _stream())
        for l in range(self.blocks):
            self.conv.forward(self.y[l], self.w[l], self.h)
            k = l + 1
            dwm.dwm_norm_join_forward(self.norm, self.drop(step, l), self.h.data_ptr(), self.z[l].data_ptr(), self.gamma[k].data_ptr(),
                                      self.beta[k].data_ptr(), self.z[k].data_ptr(), self.y[k].data_ptr(), self.mean[k].data_ptr(),
                                      self.rstd[k].data_ptr(), _stream())
        return self.y[-1]

    def backward(self, dy, step):
        """From the gradient of the last y: dw, dgamma, dbeta, and the gradient of x (returned).  Each block's gradient of its stream takes the
        place of the next one's."""
        self.dy.copy_(dy)
        for l in reversed(range(self.blocks)):
            k = l + 1
            dwm.dwm_norm_join_backward(self.norm, self.drop(step, l), self.dy.data_ptr(), None if k == self.blocks else self.dz.data_ptr(),
                                       self.z[k].data_ptr(), self.gamma[k].data_ptr(), self.mean[k].data_ptr(), self.rstd[k].data_ptr(),
                                       self.dh.data_ptr(), self.dz.data_ptr(), self.dgamma[k].data_ptr(), self.dbeta[k].data_ptr(), _stream())
            self.conv.backward(self.y[l], self.w[l], self.dh, self.dy, self.dw[l])
        # the first norm reads x, which is the stream's start too: a join without a branch
        dwm.dwm_norm_join_backward(self.norm, None, self.dy.data_ptr(), self.dz.data_ptr() if self.blocks else None, self.z[0].data_ptr(),
                                   self.gamma[0].data_ptr(), self.mean[0].data_ptr(), self.rstd[0].data_ptr(), None, self.dx.data_ptr(),
                                   self.dgamma[0].data_ptr(), self.dbeta[0].data_ptr(), _stream())
        return self.dx

    def descend(self, rate):
        for value, grad in zip(self.w + self.gamma + self.beta, self.dw + self.dgamma + self.dbeta):
            value.sub_(grad, alpha=rate)

    def close(self):
        torch.cuda.synchronize()
        self.conv.close()
        dwm.dwm_norm_plan_destroy(self.norm)


def train(net, x, target, steps, rate):
    """Mean squared errors of the steps (before each one's descent)."""
    losses = []
    for step in range(steps):
        error = net.forward(x, step) - target
        losses.append((error * error).mean())
        net.backward(error * (2.0 / error.numel()), step)
        net.descend(rate)
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 20), ("blocks", 2), ("batch", 8), ("channels", 32), ("size", 28)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--rate", type=float, default=2.0)
    a = ap.parse_args()
    net = Blocks(a.blocks, a.batch, a.channels, a.size, p=a.dropout)
    x = torch.randn(net.shape, device="cuda")
    target = torch.nn.functional.avg_pool2d(x, 5, 1, 2) * 5  # something that 7x7 filters can learn
    torch.cuda.synchronize()
    began = time.perf_counter()
    losses = train(net, x, target, a.steps, a.rate)
    torch.cuda.synchronize()
    print("mean squared error %.4f -> %.4f in %d steps, %.2f ms a step" % (losses[0], losses[-1], a.steps,
                                                                           (time.perf_counter() - began) / a.steps * 1e3))
    net.close()


if __name__ == "__main__":
    main()
