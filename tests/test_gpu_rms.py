"""Root-mean-square norms with the residual's addition through the C ABI against 64 bits: z and its checkpoint bit for bit."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
from branch_gpu import TYPE, PackedRows, Plan, Rows, n64, normal, param, ptr, stream, within

pytestmark = pytest.mark.gpu


def packed_within(packed, y, error, what):
    """Codes and scales of values known to `error`: each scale that of the block's largest, either side of a border; each code the
    nearest under it."""
    codes, scales = packed.numpy()
    packed.check()
    C = y.shape[1]
    for lo, hi in ((0, C),):
        size, e = np.abs(y[:, lo:hi]), error[:, lo:hi]
        for b in range(ref.blocks(C)):
            part, off = size[:, 32 * b:32 * b + 32], e[:, 32 * b:32 * b + 32]
            low, high = (part - off).max(axis=1), (part + off).max(axis=1)
            for r in range(len(y)):
                assert ref.scale_byte(max(low[r], 0.0)) <= scales[r, b] <= ref.scale_byte(high[r]), "%s: scale of row %d, block %d" % (what, r, b)
    within(packed.values(), y, 1.07 * error + ref.half_step(y, scales), what)


def check(rows, C, dtype, params, residual=True, from_kept=True, eps=1e-5, wide=0, off=0, kind="normal", with_dz=True, with_gamma=True, variants=None, seed=11):
    print("rms", rows, C, dtype, params, residual, from_kept, wide, off, kind, variants, flush=True)
    t = {name: Rows(rows, C, dtype, wide, off, normal(rows, C, seed + k, kind if name in ("x", "residual") else "normal") if name in ("x", "residual", "dy", "dz") else None)
         for k, name in enumerate(("x", "residual", "dy", "dz", "z", "y", "dx"))}
    gamma = param(C, params, seed + 9, 1.0) if with_gamma else None
    g64 = n64(gamma) if with_gamma else np.ones(C)
    rstd, dgamma = torch.full((rows,), float("nan"), device="cuda"), torch.full((C,), float("nan"), dtype=ref.TYPES[params], device="cuda")
    y8, kept = PackedRows(rows, C), PackedRows(rows, C)
    plan = Plan("rms", rows, C, TYPE[dtype], TYPE[params], eps, strides=t, variants=variants)
    try:
        dwm.dwm_rms_forward(plan.plan, t["x"].ptr(), t["residual"].ptr() if residual else None, ptr(gamma), t["z"].ptr() if residual else None, t["y"].ptr(), y8.t,
                            kept.t, ptr(rstd), stream())
        z32 = t["x"].numpy().astype(np.float32)
        if residual:
            want = ref.rounded(t["residual"].numpy().astype(np.float32) + z32, dtype)
            assert torch.equal(t["z"].view.cpu(), want)
            z32 = want.float().numpy()
        codes, scales = kept.numpy()
        same = ref.pack(z32)
        assert np.array_equal(scales, same[1]) and ref.same_codes(codes, same[0])
        kept.check()
        z = z32.astype(np.float64)
        y64, r64 = ref.rms(z, g64, eps)
        t_raw, t_y, t_rstd = ref.rms_tolerance(z, g64, eps, dtype)
        within(n64(rstd), r64, t_rstd, "rstd")
        within(t["y"].numpy(), y64, t_y, "y")
        packed_within(y8, y64, t_raw, "y in 8 bits")
        source = t["z"] if residual else t["x"]
        if not from_kept:
            dwm.dwm_rms_set_stride(plan.plan, "z", source.stride)
        dwm.dwm_rms_backward(plan.plan, t["dy"].ptr(), t["dz"].ptr() if with_dz else None, None if from_kept else source.ptr(), kept.t if from_kept else None,
                             ptr(gamma), ptr(rstd), t["dx"].ptr(), ptr(dgamma), stream())
        at = kept.values() if from_kept else z
        dy, dz = t["dy"].numpy(), t["dz"].numpy() if with_dz else np.zeros((rows, C))
        dx64, dg64 = ref.rms_backward(dy, dz, at, g64, n64(rstd))
        t_dx, t_dg = ref.rms_backward_tolerance(dy, dz, at, g64, n64(rstd), dtype, params)
        within(t["dx"].numpy(), dx64, t_dx, "dx")
        within(n64(dgamma), dg64, t_dg, "dgamma")
        assert all(v.untouched() for v in t.values())
    finally:
        plan.close()


@pytest.mark.parametrize("dtype, params", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_types(dtype, params):
    check(37, 1021, dtype, params, wide=5, off=3)
    check(70, 4096, dtype, params, from_kept=False)


@pytest.mark.parametrize("rows, C", [(1, 1), (1, 4096), (3, 7), (5, 31), (130, 32), (9, 33), (300, 64), (40, 100), (33, 256), (17, 500), (6, 1000), (5, 2047), (4, 2049),
                                     (3, 8192), (3, 8200), (2, 16384), (2, 16385), (2, 40000), (2100, 24), (2100, 520), (2049, 1025)])
def test_sizes(rows, C):
    check(rows, C, "bf16", "f32", from_kept=C % 2 == 0)
    check(rows, C, "f32", "f32", residual=C % 3 != 0, from_kept=C % 2 == 1, wide=1)


@pytest.mark.parametrize("variant", range(15))
def test_variants(variant):
    fits = 8 * [16384, 4, 8, 16, 32, 64, 128, 128, 256, 256, 512, 512, 1024, 1024, 2048][variant]
    for C in sorted({min(fits, 1000), min(fits, 16384) - 3}):
        check(21, C, "bf16", "bf16", variants={"forward": variant, "backward": variant}, from_kept=variant % 2 == 0)


@pytest.mark.parametrize("kind", ["small", "outlier", "spread"])
def test_values(kind):
    check(20, 700, "f32", "f32", kind=kind, eps=1e-6)
    check(20, 700, "bf16", "f32", kind=kind, with_dz=False, with_gamma=False)
    check(20, 700, "f32", "f32", kind=kind, eps=0.0, residual=False, from_kept=False)


def test_rows_of_zeros_and_rows_that_are_not_finite():
    rows, C = 6, 200
    v = normal(rows, C, 1)
    v[1], v[2, 5], v[4, 7] = 0.0, np.inf, np.nan
    x, y, y8, kept = Rows(rows, C, "f32", values=v), Rows(rows, C, "f32"), PackedRows(rows, C), PackedRows(rows, C)
    rstd = torch.empty(rows, device="cuda")
    for variant in (-1, 0):
        plan = Plan("rms", rows, C, dwm.DWM_F32, dwm.DWM_F32, 1e-5, variants={"forward": variant})
        dwm.dwm_rms_forward(plan.plan, x.ptr(), None, None, None, y.ptr(), y8.t, kept.t, ptr(rstd), stream())
        torch.cuda.synchronize()
        good = [0, 1, 3, 5]
        want, r = ref.rms(v[good].astype(np.float64), np.ones(C), 1e-5)
        raw, t_y, _ = ref.rms_tolerance(v[good].astype(np.float64), np.ones(C), 1e-5, "f32")
        within(y.numpy()[good], want, t_y, "y")
        assert np.isnan(y.numpy()[4]).all() and np.isnan(y.numpy()[2, 5]) and not y.numpy()[2, :5].any()
        assert not y8.values()[1].any() and np.array_equal(np.isnan(kept.values()), ~np.isfinite(v))
        y8.check()
        plan.close()


def test_zero_rstd_without_eps():
    """A row of zeros with eps = 0 has an infinite rstd and y is NaN; nothing behind the row's channels changes, no other row."""
    v = normal(3, 37, 1)
    v[1] = 0
    x, y, y8 = Rows(3, 37, "f16", values=v), Rows(3, 37, "f16"), PackedRows(3, 37)
    plan = Plan("rms", 3, 37, dwm.DWM_F16, dwm.DWM_F16, 0.0)
    dwm.dwm_rms_forward(plan.plan, x.ptr(), None, None, None, y.ptr(), y8.t, None, None, stream())
    torch.cuda.synchronize()
    y8.check()
    assert np.isnan(y.numpy()[1]).all() and np.isfinite(y.numpy()[[0, 2]]).all() and np.isnan(y8.values()[1]).all()
    plan.close()


def test_parts_of_a_call_and_outputs_in_place():
    for C in (300, 20000):
        rows = 9
        v, r, g, d = (normal(rows, C, k) for k in range(4))
        gamma = param(C, "f32", 5, 1.0)

        def tensors():
            return [Rows(rows, C, "bf16", values=a) for a in (v, r, g, d)]

        x, res, dy, dz = tensors()
        z, y, dx = (Rows(rows, C, "bf16") for _ in range(3))
        rstd, only, dgamma, sums = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        plan = Plan("rms", rows, C, dwm.DWM_BF16, dwm.DWM_F32, 1e-5)
        f, b = dwm.dwm_rms_forward, dwm.dwm_rms_backward
        f(plan.plan, x.ptr(), res.ptr(), ptr(gamma), z.ptr(), y.ptr(), None, None, ptr(rstd), stream())
        f(plan.plan, x.ptr(), res.ptr(), None, None, None, None, None, ptr(only), stream())
        assert torch.equal(rstd, only)
        x2, res2, dy2, dz2 = tensors()
        f(plan.plan, x2.ptr(), res2.ptr(), ptr(gamma), res2.ptr(), x2.ptr(), None, None, None, stream())
        assert torch.equal(res2.view, z.view) and torch.equal(x2.view, y.view)
        x2, res2, dy2, dz2 = tensors()
        f(plan.plan, x2.ptr(), res2.ptr(), ptr(gamma), x2.ptr(), None, None, None, None, stream())
        assert torch.equal(x2.view, z.view)
        b(plan.plan, dy.ptr(), dz.ptr(), z.ptr(), None, ptr(gamma), ptr(rstd), dx.ptr(), ptr(dgamma), stream())
        b(plan.plan, dy.ptr(), None, z.ptr(), None, ptr(gamma), ptr(rstd), None, ptr(sums), stream())
        assert torch.equal(dgamma, sums)
        b(plan.plan, dy2.ptr(), dz2.ptr(), z.ptr(), None, ptr(gamma), ptr(rstd), dy2.ptr(), ptr(sums), stream())
        assert torch.equal(dy2.view, dx.view) and torch.equal(dgamma, sums)
        b(plan.plan, dy.ptr(), dz2.ptr(), z.ptr(), None, ptr(gamma), ptr(rstd), dz2.ptr(), None, stream())
        assert torch.equal(dz2.view, dx.view)
        plan.close()


def test_no_rows():
    plan = Plan("rms", 0, 100, dwm.DWM_BF16, dwm.DWM_BF16, 1e-5)
    dgamma = torch.full((100,), float("nan"), dtype=torch.bfloat16, device="cuda")
    dwm.dwm_rms_forward(plan.plan, None, None, None, None, None, None, None, None, stream())
    dwm.dwm_rms_backward(plan.plan, None, None, None, None, None, None, None, ptr(dgamma), stream())
    torch.cuda.synchronize()
    assert not dgamma.any()
    plan.close()
