"""Rows in 8 bits and activations with their checkpoints through the C ABI: codes and scales bit for bit, values against 64 bits."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
from branch_gpu import ACT, TYPE, PackedRows, Plan, Rows, n64, normal, param, ptr, stream, within

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 129), (7, 1021), (64, 784), (9, 2048), (3, 2049), (2, 5000), (300, 40)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, C", SIZES)
def test_pack_and_unpack(rows, C, dtype):
    for wide, off in ((0, 0), (5, 3)):
        print("pack", rows, C, dtype, wide, off, flush=True)
        x = Rows(rows, C, dtype, wide, off, normal(rows, C, 1, "spread" if dtype != "f16" else "normal"))
        want = ref.pack(x.view.float().cpu().numpy())
        packed = PackedRows(rows, C)
        dwm.dwm_pack(TYPE[dtype], rows, C, x.ptr(), x.stride, packed.t, stream())
        codes, scales = packed.numpy()
        assert np.array_equal(scales, want[1]) and ref.same_codes(codes, want[0])
        packed.check()
        y = Rows(rows, C, dtype, wide, off)
        dwm.dwm_unpack(TYPE[dtype], rows, C, packed.t, y.ptr(), y.stride, stream())
        torch.cuda.synchronize()
        assert torch.equal(y.view.cpu(), torch.from_numpy(ref.unpack(codes, scales, C)).to(ref.TYPES[dtype]))
        assert y.untouched() and x.untouched()


def test_values_at_the_borders():
    tiny = 2.0 ** -149
    rows = [[448.0, 1.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 17.0, 18.0, 19.0],  # ties, the smallest code, the largest
            [448.00003, 449.0, 1.0, -448.0, 224.0, 0.0, -0.0, 3.0],  # just over: the next scale
            [447.99997, 224.00002, 232.0, 240.0, 248.0, 8.5, 9.5, 10.5],
            [0.0, -0.0, 0, 0, 0, 0, 0, 0],
            [tiny, -tiny, 100 * tiny, 0, 0, 0, 0, 2.0 ** -126],  # below the smallest scale
            [448 * 2.0 ** -127, 2.0 ** -136, 2.0 ** -137, 1.5 * 2.0 ** -136, 0, 0, 0, 0],
            [3.4e38, -3.4e38, 1.0, 1e30, 1e36, 0, 0, 0],
            [np.inf, 1.0, 2.0, -np.inf, np.nan, 3.0, 0.5, -1.0],  # their own elements alone
            [np.inf] * 8, [np.nan] * 8, [np.inf, 3.4e38, 0, 0, 0, 0, 0, 0]]
    v = np.zeros((len(rows), 40), np.float32)
    v[:, :8] = rows
    v[:, 32:] = 5.0  # a block that nothing of this reaches
    want = ref.pack(v)
    x, packed, y = Rows(len(rows), 40, "f32", values=v), PackedRows(len(rows), 40), Rows(len(rows), 40, "f32")
    dwm.dwm_pack(dwm.DWM_F32, len(rows), 40, x.ptr(), x.stride, packed.t, stream())
    dwm.dwm_unpack(dwm.DWM_F32, len(rows), 40, packed.t, y.ptr(), y.stride, stream())
    torch.cuda.synchronize()
    codes, scales = packed.numpy()
    assert np.array_equal(scales, want[1]) and ref.same_codes(codes, want[0])
    packed.check()
    with np.errstate(over="ignore"):
        values = ref.unpack(*want, 40).astype(np.float32)
    assert np.array_equal(y.view.cpu().numpy(), values, equal_nan=True)


def test_every_code_comes_back():
    codes = np.tile(np.arange(256, dtype=np.uint8), (3, 1))
    packed = PackedRows(3, 256)
    packed.c[:packed.nc] = torch.from_numpy(codes.reshape(-1)).cuda()
    scales = np.array([[0] * 8, [127] * 8, [1, 2, 60, 126, 128, 200, 246, 247]], np.uint8)
    packed.s[:packed.ns] = torch.from_numpy(scales.reshape(-1)).cuda()
    y = Rows(3, 256, "f32")
    dwm.dwm_unpack(dwm.DWM_F32, 3, 256, packed.t, y.ptr(), y.stride, stream())
    torch.cuda.synchronize()
    with np.errstate(over="ignore"):
        assert np.array_equal(y.view.cpu().numpy(), ref.unpack(codes, scales, 256).astype(np.float32), equal_nan=True)


def check(act, rows, C, dtype, params, with_bias=True, wide=0, off=0, kind="normal", seed=5):
    print("act", act, rows, C, dtype, params, with_bias, wide, off, kind, flush=True)
    x, dy = (Rows(rows, C, dtype, wide, off, normal(rows, C, seed + k, kind if k == 0 else "normal") * (3 if k == 0 else 1)) for k in range(2))
    y, dx, dx2 = (Rows(rows, C, dtype, wide, off) for _ in range(3))
    bias = param(C, params, seed + 3) if with_bias else None
    kept = PackedRows(rows, C)
    dbias, dbias2 = (torch.full((C,), float("nan"), dtype=ref.TYPES[params], device="cuda") for _ in range(2))
    plan = Plan("act", ACT[act], rows, C, TYPE[dtype], TYPE[params], strides={"x": x, "y": y, "dy": dy, "dx": dx})
    try:
        dwm.dwm_act_forward(plan.plan, x.ptr(), ptr(bias), y.ptr(), kept.t, stream())
        dwm.dwm_act_backward(plan.plan, dy.ptr(), None, None, kept.t, dx.ptr(), ptr(dbias), stream())
        dwm.dwm_act_backward(plan.plan, dy.ptr(), x.ptr(), ptr(bias), None, dx2.ptr(), ptr(dbias2), stream())
        p32 = x.numpy().astype(np.float32) + (n64(bias).astype(np.float32) if with_bias else np.float32(0))
        p = p32.astype(np.float64)
        codes, scales = kept.numpy()
        want = ref.pack(p32)
        assert np.array_equal(scales, want[1]) and ref.same_codes(codes, want[0])
        kept.check()
        within(y.numpy(), ref.act(act, p), ref.act_error(act, p) + ref.stored(ref.act(act, p), dtype), "y")
        for at, out, sums in ((kept.values(), dx, dbias), (p, dx2, dbias2)):
            g = dy.numpy() * ref.slope(act, at)
            e = np.abs(dy.numpy()) * ref.slope_error(act, at) + 2.0 ** -24 * np.abs(g)
            within(out.numpy(), g, e + ref.stored(g, dtype), "dx")
            total = g.sum(axis=0)
            within(n64(sums), total, e.sum(axis=0) + ref.rows_error(np.abs(g)) + ref.stored(total, params), "dbias")
        assert all(t.untouched() for t in (x, dy, y, dx, dx2))
    finally:
        plan.close()


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype, params", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_activations(act, dtype, params):
    check(act, 37, 1021, dtype, params)
    check(act, 5, 4096, dtype, params, wide=11, off=3)


@pytest.mark.parametrize("rows, C", SIZES + [(5000, 96), (3000, 9)])
def test_activation_sizes(rows, C):
    check("gelu", rows, C, "bf16", "f32", wide=8)
    check("silu", rows, C, "f32", "f32", with_bias=False)


def test_activation_of_small_and_large_values():
    for act in ref.ACTS:
        for kind in ("small", "spread", "outlier"):
            check(act, 40, 300, "f32", "f32", kind=kind)


def test_parts_of_a_call():
    """Each output alone, in place, and the sums of dy's rows without an activation."""
    rows, C = 70, 200
    v, g = normal(rows, C, 1), normal(rows, C, 2)
    plan = Plan("act", dwm.DWM_ACT_SILU, rows, C, dwm.DWM_F16, dwm.DWM_F32)
    bias = param(C, "f32", 3)
    x, y, dy, dx = Rows(rows, C, "f16", values=v), Rows(rows, C, "f16"), Rows(rows, C, "f16", values=g), Rows(rows, C, "f16")
    kept, alone = PackedRows(rows, C), PackedRows(rows, C)
    dbias, other = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    dwm.dwm_act_forward(plan.plan, x.ptr(), ptr(bias), y.ptr(), kept.t, stream())
    dwm.dwm_act_forward(plan.plan, x.ptr(), ptr(bias), None, alone.t, stream())
    assert torch.equal(kept.c, alone.c) and torch.equal(kept.s, alone.s)
    again = Rows(rows, C, "f16", values=v)
    dwm.dwm_act_forward(plan.plan, again.ptr(), ptr(bias), again.ptr(), None, stream())
    assert torch.equal(again.view, y.view)
    dwm.dwm_act_backward(plan.plan, dy.ptr(), None, None, kept.t, dx.ptr(), ptr(dbias), stream())
    dwm.dwm_act_backward(plan.plan, dy.ptr(), None, None, kept.t, None, ptr(other), stream())
    assert torch.equal(dbias, other)
    again = Rows(rows, C, "f16", values=g)
    dwm.dwm_act_backward(plan.plan, again.ptr(), None, None, kept.t, again.ptr(), ptr(other), stream())
    assert torch.equal(again.view, dx.view) and torch.equal(dbias, other)
    plan.close()
    plan = Plan("act", dwm.DWM_ACT_NONE, rows, C, dwm.DWM_F16, dwm.DWM_F32)
    dwm.dwm_act_backward(plan.plan, dy.ptr(), None, None, None, None, ptr(other), stream())
    within(n64(other), dy.numpy().sum(axis=0), ref.rows_error(np.abs(dy.numpy())), "dbias")
    plan.close()


def test_no_rows():
    plan = Plan("act", dwm.DWM_ACT_GELU, 0, 100, dwm.DWM_BF16, dwm.DWM_F32)
    dbias = torch.full((100,), float("nan"), device="cuda")
    dwm.dwm_act_forward(plan.plan, None, None, None, None, stream())
    dwm.dwm_act_backward(plan.plan, None, None, None, None, None, ptr(dbias), stream())
    torch.cuda.synchronize()
    assert not dbias.any()
    plan.close()
    dwm.dwm_pack(dwm.DWM_F32, 0, 5, None, 5, None, stream())


def test_nan_and_infinity():
    v = normal(4, 64, 1)
    v[1, 3], v[2, 40], v[3, 0] = np.nan, np.inf, -np.inf
    for act in ref.ACTS:
        x, y, kept = Rows(4, 64, "f32", values=v), Rows(4, 64, "f32"), PackedRows(4, 64)
        dx = Rows(4, 64, "f32")
        plan = Plan("act", ACT[act], 4, 64, dwm.DWM_F32, dwm.DWM_F32)
        dwm.dwm_act_forward(plan.plan, x.ptr(), None, y.ptr(), kept.t, stream())
        dwm.dwm_act_backward(plan.plan, x.ptr(), None, None, kept.t, dx.ptr(), None, stream())
        torch.cuda.synchronize()
        fine = np.isfinite(v)
        assert np.isfinite(y.view.cpu().numpy()[fine]).all() and np.isfinite(dx.view.cpu().numpy()[fine]).all()
        assert np.isnan(y.view.cpu().numpy()[1, 3]) and np.isnan(dx.view.cpu().numpy()[1, 3])
        assert np.array_equal(np.isnan(kept.values()), ~fine)
        plan.close()
