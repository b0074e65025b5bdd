"""Norms of so many rows that workgroups go on to further ones, the next already on its way: every row, rows over several waves, parts of groups at the end, in place."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
import rows_exact as exact
from branch_gpu import TYPE, PackedRows, Plan, Rows, n64, param, ptr, stream, within

pytestmark = pytest.mark.gpu

# Threads of a row: 512, 256, 128 (two rows to a workgroup, the last one alone), 1024, 64, 16.  Workgroups stay from 4096 of 256 threads on, 2048 of 512, 1024 of 1024.
SIZES = [(2101, 4096), (4103, 2048), (8197, 1000), (1030, 8192), (17001, 500), (66001, 100)]


def same(packed, v, what):
    packed.check()
    codes, scales = packed.numpy()
    want = exact.pack(v)
    assert np.array_equal(scales, want[1]) and np.array_equal(codes, want[0]), what


@pytest.mark.parametrize("dtype, params", [("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("rows, C", SIZES)
def test_every_row(rows, C, dtype, params):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, res, dy, dz, z, y, dx = (Rows(rows, C, dtype, wide, 0) for wide in (0, 8, 3, 0, 5, 0, 8))
    for t in (x, res, dy, dz):
        t.view.copy_(torch.randn(rows, C, generator=g, device="cuda"))
    gamma, eps = param(C, params, 9, 1.0), 1e-5
    y8, kept, rstd, dgamma = PackedRows(rows, C), PackedRows(rows, C), torch.empty(rows, device="cuda"), torch.empty(C, dtype=ref.TYPES[params], device="cuda")
    plan = Plan("rms", rows, C, TYPE[dtype], TYPE[params], eps, strides={"x": x, "residual": res, "dy": dy, "z": z, "dx": dx})
    dwm.dwm_rms_forward(plan.plan, x.ptr(), res.ptr(), ptr(gamma), z.ptr(), y.ptr(), y8.t, kept.t, ptr(rstd), stream())
    dwm.dwm_rms_backward(plan.plan, dy.ptr(), dz.ptr(), None, kept.t, ptr(gamma), ptr(rstd), dx.ptr(), ptr(dgamma), stream())
    torch.cuda.synchronize()
    joined = (res.view.float() + x.view.float()).to(ref.TYPES[dtype])
    assert torch.equal(z.view, joined)
    z64, g64 = joined.double().cpu().numpy(), n64(gamma)
    want, root = exact.norm(z64, g64, eps)
    within(n64(rstd), root, exact.one_rounding(root), "rstd")
    within(y.numpy(), want, exact.one_rounding(want) + ref.stored(want, dtype), "y")
    same(kept, z64, "kept")
    same(y8, want, "y in 8 bits")
    at, dy64, dz64 = kept.values(), dy.numpy(), dz.numpy()
    dx64, dg64 = ref.rms_backward(dy64, dz64, at, g64, n64(rstd))
    t_dx, t_dg = ref.rms_backward_tolerance(dy64, dz64, at, g64, n64(rstd), dtype, params)
    within(dx.numpy(), dx64, t_dx, "dx")
    within(n64(dgamma), dg64, t_dg, "dgamma")
    assert all(t.untouched() for t in (x, res, dy, dz, z, y, dx))
    # in place: z over the residual and y over x, z over x, dx over dy and over dz
    plan.close()
    plan = Plan("rms", rows, C, TYPE[dtype], TYPE[params], eps, strides={"x": x, "residual": res, "dy": dy, "z": res, "y": x, "dx": dy})
    x_was, res_was, dz_was = x.view.clone(), res.view.clone(), dz.view.clone()
    dwm.dwm_rms_forward(plan.plan, x.ptr(), res.ptr(), ptr(gamma), res.ptr(), x.ptr(), None, None, None, stream())
    assert torch.equal(res.view, joined) and torch.equal(x.view, y.view)
    x.view.copy_(x_was)
    res.view.copy_(res_was)
    dwm.dwm_rms_set_stride(plan.plan, "z", x.stride)
    dwm.dwm_rms_forward(plan.plan, x.ptr(), res.ptr(), ptr(gamma), x.ptr(), None, None, None, None, stream())
    assert torch.equal(x.view, joined)
    dwm.dwm_rms_backward(plan.plan, dy.ptr(), dz.ptr(), None, kept.t, ptr(gamma), ptr(rstd), dy.ptr(), None, stream())
    assert torch.equal(dy.view, dx.view)
    dy.view.copy_(torch.from_numpy(dy64))
    dwm.dwm_rms_set_stride(plan.plan, "dx", dz.stride)
    dwm.dwm_rms_backward(plan.plan, dy.ptr(), dz.ptr(), None, kept.t, ptr(gamma), ptr(rstd), dz.ptr(), None, stream())
    assert torch.equal(dz.view, dx.view) and not torch.equal(dz_was, dx.view)
    plan.close()
