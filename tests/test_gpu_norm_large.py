"""Joins, gradients and the sums of the parameters' gradients over tensors of more than 2^31 elements, in every kind of kernel: masks by the places of
the last elements, values at the last positions, sums to which only those contribute.  Bounds of norm_reference.py."""
import numpy as np
import pytest
import torch

import norm_reference as ref
import paper_2002_00552_amd as dwm

pytestmark = pytest.mark.gpu

TAIL = 4
EPS = 1e-5
SEED, SEQUENCE, P = 0x1234567890ABCDEF, 77, 0.3


def _within(got, want, tolerance, what):
    worst = np.abs(got - want) - tolerance
    assert np.isfinite(got).all() and (worst <= 0).all(), "%s: off by %.3g, %.3g allowed" % (
        what, np.abs(got - want).flat[worst.argmax()], np.broadcast_to(tolerance, want.shape).flat[worst.argmax()])


def _values(shape, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


class Large:
    """A bfloat16 tensor of one value, but for the last positions; `stride` elements from one o to the next."""

    def __init__(self, shape, value, seed=None, stride=None):
        outer, C, inner = shape
        self.rows = inner == 1
        self.buffer = torch.empty((outer, stride or C * inner), dtype=torch.bfloat16, device="cuda").fill_(value)
        self.view = self.buffer[:, :C * inner].unflatten(1, (C, inner))
        if seed is not None:
            self.tail().copy_(_values(self.tail().shape, seed))

    def tail(self):
        return self.view[-TAIL:] if self.rows else self.view[-1:, :, -TAIL:]

    def numpy(self):
        return self.tail().double().cpu().numpy()

    def ptr(self):
        return self.buffer.data_ptr()


def _kept_tail(shape):
    """Which elements of the last positions a mask keeps, from their places in the dense order."""
    outer, C, inner = shape
    limit = np.uint64(round(P * 2.0 ** 32))
    if inner == 1:
        return (ref.words(TAIL * C, SEED, SEQUENCE, (outer - TAIL) * C) >= limit).reshape(TAIL, C, 1)
    first = [((outer - 1) * C + c) * inner + inner - TAIL for c in range(C)]
    return np.stack([ref.words(TAIL, SEED, SEQUENCE, f) >= limit for f in first])[None]


@pytest.mark.parametrize("variant", [-1, 0])
@pytest.mark.parametrize("shape, stride", [((1 << 20, 2056, 1), None), ((3, 8, 100_000_007), None), ((1 << 19, 264, 1), 8208), ((5, 24, 900), 1 << 29)],
                         ids=["rows", "maps", "rows-apart", "maps-apart"])
def test_joins_and_gradients_beyond_32_bits(shape, stride, variant):
    outer, C, inner = shape
    print(shape, stride, variant, flush=True)
    rng = np.random.default_rng(3)
    gamma = torch.from_numpy((1 + 0.5 * rng.standard_normal(C)).astype(np.float32)).cuda()
    beta = torch.from_numpy((0.5 * rng.standard_normal(C)).astype(np.float32)).cuda()
    g64, b64 = gamma.double().cpu().numpy(), beta.double().cpu().numpy()
    dgamma, dbeta = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    mean, rstd = (torch.full((outer, inner), float("nan"), device="cuda") for _ in range(2))
    drop = dwm.dwm_dropout_t(P, SEED, SEQUENCE, None)
    plan = dwm.dwm_norm_plan_create(outer, C, inner, dwm.DWM_BF16, dwm.DWM_F32, EPS)
    try:
        for stage in ("forward", "backward"):
            dwm.dwm_norm_set_variant(plan, stage, variant)
        for name in ("residual", "z", "dy", "dx") if stride else ():
            dwm.dwm_norm_set_stride(plan, name, stride)
        ws = torch.empty(max(dwm.dwm_norm_workspace_bytes(plan), 256), dtype=torch.uint8, device="cuda")
        dwm.dwm_norm_set_workspace(plan, ws.data_ptr(), ws.numel())
        st = torch.cuda.current_stream().cuda_stream
        x, z, y = Large(shape, 0.5, 11), Large(shape, 1.0, 12, stride), Large(shape, 0.0)
        branch = ref.dropout32(x.numpy().astype(np.float32), _kept_tail(shape), P)
        want = ref.rounded(z.numpy().astype(np.float32) + branch, "bf16")
        dwm.dwm_norm_join_forward(plan, drop, x.ptr(), z.ptr(), gamma.data_ptr(), beta.data_ptr(), z.ptr(), y.ptr(), mean.data_ptr(), rstd.data_ptr(), st)
        assert torch.equal(z.tail().cpu(), want)
        z64 = z.numpy()
        t_y, t_mean, t_rstd = ref.tolerances_forward(z64, g64, b64, EPS, "bf16")
        want_y, want_mean, want_rstd = ref.norm(z64, g64, b64, EPS)
        _within(y.numpy(), want_y, t_y, "y")
        last = (slice(-TAIL, None), slice(None)) if inner == 1 else (slice(-1, None), slice(-TAIL, None))
        m, r = mean[last].double().cpu().numpy(), rstd[last].double().cpu().numpy()
        _within(m, want_mean, t_mean, "mean")
        _within(r, want_rstd, t_rstd, "rstd")
        del x, y
        # dx in dy's memory, dresidual in dz's; only the last positions have a gradient of y
        dy, dz = Large(shape, 0.0, 13, stride), Large(shape, 0.25, 14)
        dy64, dz64 = dy.numpy(), dz.numpy()
        dwm.dwm_norm_join_backward(plan, drop, dy.ptr(), dz.ptr(), z.ptr(), gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dy.ptr(), dz.ptr(),
                                   dgamma.data_ptr(), dbeta.data_ptr(), st)
        want, want_dgamma, want_dbeta = ref.norm_backward(dy64, z64, g64, m, r)
        want = want + dz64
        t_dx, t_dgamma, t_dbeta = ref.tolerances_backward(dy64, z64, g64, m, r, dz64, want, "bf16", "f32", want_dgamma, want_dbeta)
        _within(dz.numpy(), want, t_dx, "dresidual")
        keep, s = _kept_tail(shape), float(ref.scale(P))
        _within(dy.numpy(), np.where(keep, want * s, 0.0), np.where(keep, t_dx * s * 1.01 + ref.TINY["bf16"], 0.0), "dx")
        _within(dgamma.double().cpu().numpy(), want_dgamma, t_dgamma, "dgamma")
        _within(dbeta.double().cpu().numpy(), want_dbeta, t_dbeta, "dbeta")
        # elsewhere dresidual is what came along the stream
        assert bool((dz.view[0, :, :1] == 0.25).all())
    finally:
        torch.cuda.synchronize()
        dwm.dwm_norm_plan_destroy(plan)
