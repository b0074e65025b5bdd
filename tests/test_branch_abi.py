"""What the entry points over rows (rows in 8 bits, root-mean-square norms, activations, matrix products) refuse, and what their
plans say; no GPU is needed, nothing is launched."""
import ctypes
import math

import pytest

import paper_2002_00552_amd as dwm

ONE = 4096  # an address no call reads
BAD = dwm.DWM_ERR_INVALID_ARG
P = dwm.dwm_packed_t


def _refused(status, fn, *args):
    with pytest.raises(dwm.DwmError) as e:
        fn(*args)
    assert e.value.status == status


def test_packed_sizes():
    assert dwm.dwm_packed_codes_bytes(3, 1) == 96 and dwm.dwm_packed_scales_bytes(3, 1) == 12
    assert dwm.dwm_packed_codes_bytes(3, 128) == 384 and dwm.dwm_packed_scales_bytes(3, 128) == 12
    assert dwm.dwm_packed_codes_bytes(5, 129) == 800 and dwm.dwm_packed_scales_bytes(5, 129) == 40
    assert dwm.dwm_packed_codes_bytes(0, 8) == 0 and dwm.dwm_packed_codes_bytes(-1, 8) == 0 and dwm.dwm_packed_codes_bytes(8, 0) == 0
    assert dwm.dwm_packed_codes_bytes(1, (1 << 20) + 1) == 0 and dwm.dwm_packed_scales_bytes(1 << 40, 2) == 0
    assert dwm.dwm_packed_codes_bytes(1 << 20, 1 << 20) == 1 << 40


@pytest.mark.parametrize("fn", [dwm.dwm_pack, dwm.dwm_unpack])
@pytest.mark.parametrize("type, rows, C, x, stride, packed, status", [
    (dwm.DWM_PACKED, 1, 8, ONE, 8, P(ONE, ONE), BAD),
    (-1, 1, 8, ONE, 8, P(ONE, ONE), BAD),
    (0, -1, 8, ONE, 8, P(ONE, ONE), BAD),
    (0, 1, 0, ONE, 8, P(ONE, ONE), BAD),
    (0, 1, 8, ONE, 7, P(ONE, ONE), BAD),
    (0, 1, 8, None, 8, P(ONE, ONE), BAD),
    (0, 1, 8, ONE + 2, 8, P(ONE, ONE), BAD),
    (1, 1, 8, ONE + 1, 8, P(ONE, ONE), BAD),
    (0, 1, 8, ONE, 8, None, BAD),
    (0, 1, 8, ONE, 8, P(None, ONE), BAD),
    (0, 1, 8, ONE, 8, P(ONE, None), BAD),
    (0, 1, 8, ONE, 8, P(ONE + 8, ONE), BAD),
    (0, 1, 8, ONE, 8, P(ONE, ONE + 2), BAD),
    (0, 1, (1 << 20) + 1, ONE, 1 << 21, P(ONE, ONE), dwm.DWM_ERR_UNSUPPORTED),
    (0, 1 << 40, 2, ONE, 2, P(ONE, ONE), dwm.DWM_ERR_UNSUPPORTED),
    (0, 1 << 30, 2, ONE, 1 << 20, P(ONE, ONE), dwm.DWM_ERR_UNSUPPORTED),
])
def test_pack_refuses(fn, type, rows, C, x, stride, packed, status):
    args = (type, rows, C, x, stride, packed) if fn is dwm.dwm_pack else (type, rows, C, packed, x, stride)
    _refused(status, fn, *args)


@pytest.mark.parametrize("args, status", [
    ((-1, 8, 0, 0, 1e-5), BAD), ((1, 0, 0, 0, 1e-5), BAD), ((1, 8, 3, 0, 1e-5), BAD), ((1, 8, 3, 3, 1e-5), BAD), ((1, 8, -1, 0, 1e-5), BAD),
    ((1, 8, dwm.DWM_F16, dwm.DWM_BF16, 1e-5), BAD), ((1, 8, dwm.DWM_F32, dwm.DWM_F16, 1e-5), BAD),
    ((1, 8, 0, 0, -1e-9), BAD), ((1, 8, 0, 0, math.nan), BAD), ((1, 8, 0, 0, math.inf), BAD),
    ((1, (1 << 20) + 1, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED), (((1 << 63) - 1, 2, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED),
])
def test_rms_plans_that_are_refused(args, status):
    _refused(status, dwm.dwm_rms_plan_create, *args)


@pytest.mark.parametrize("args, status", [
    ((4, 1, 8, 0, 0), BAD), ((-1, 1, 8, 0, 0), BAD), ((0, -1, 8, 0, 0), BAD), ((0, 1, 0, 0, 0), BAD), ((0, 1, 8, 3, 0), BAD), ((0, 1, 8, 1, 2), BAD),
    ((0, 1, (1 << 20) + 1, 0, 0), dwm.DWM_ERR_UNSUPPORTED), ((0, 1 << 40, 2, 0, 0), dwm.DWM_ERR_UNSUPPORTED),
])
def test_act_plans_that_are_refused(args, status):
    _refused(status, dwm.dwm_act_plan_create, *args)


F32, F16, BF16, PACKED = dwm.DWM_F32, dwm.DWM_F16, dwm.DWM_BF16, dwm.DWM_PACKED
OUT = dwm.DWM_ERR_UNSUPPORTED


@pytest.mark.parametrize("args, status", [
    ((-1, 8, 8, F16, F16, F32, 0, 0), BAD), ((8, -1, 8, F16, F16, F32, 0, 0), BAD), ((8, 8, -1, F16, F16, F32, 0, 0), BAD),
    ((8, 8, 8, 4, F16, F32, 0, 0), BAD), ((8, 8, 8, F16, PACKED, F32, 0, 0), BAD), ((8, 8, 8, F16, F16, BF16, 0, 0), BAD),
    ((8, 8, 8, PACKED, BF16, F16, 0, 0), BAD), ((8, 8, 8, F16, F16, F32, 4, 0), BAD), ((8, 8, 8, F16, F16, F32, 0, 4), BAD),
    ((8, 8, 8, F16, F16, F32, 0, -1), BAD),
    ((8, 8, 8, F32, F32, F32, 0, 0), OUT), ((8, 8, 8, F16, BF16, F32, 0, 0), OUT), ((8, 8, 8, PACKED, F32, F32, 0, 0), OUT),
    ((8, 8, 8, PACKED, F16, F32, 0, 1), OUT), (((1 << 24) + 1, 8, 8, F16, F16, F32, 0, 0), OUT), ((8, (1 << 24) + 1, 8, F16, F16, F32, 0, 0), OUT),
    ((8, 8, (1 << 24) + 1, F16, F16, F32, 0, 0), OUT), ((1 << 24, 1 << 14, 8, F16, F16, F32, 0, 0), OUT),
])
def test_matmul_plans_that_are_refused(args, status):
    _refused(status, dwm.dwm_matmul_plan_create, *args)


@pytest.fixture
def rms():
    p = dwm.dwm_rms_plan_create(4, 96, F16, F32, 1e-5)
    yield p
    dwm.dwm_rms_plan_destroy(p)


@pytest.fixture
def act():
    p = dwm.dwm_act_plan_create(dwm.DWM_ACT_GELU, 4, 96, F16, F32)
    yield p
    dwm.dwm_act_plan_destroy(p)


def test_null_plans_are_refused():
    L = dwm.lib()
    for family in ("rms", "act", "matmul"):
        f = lambda name: getattr(L, "dwm_%s_%s" % (family, name))  # noqa: E731
        assert f("plan_destroy")(None) == BAD and f("workspace_bytes")(None) == 0
        assert f("set_workspace")(None, ONE, 1 << 20) == BAD and f("set_stride")(None, b"x", 1) == BAD
    assert L.dwm_rms_plan_create(None, 1, 1, 0, 0, 1e-5) == BAD and L.dwm_act_plan_create(None, 0, 1, 1, 0, 0) == BAD
    assert L.dwm_matmul_plan_create(None, 1, 1, 1, 1, 1, 0, 0, 0) == BAD
    assert L.dwm_rms_plan_info(None, ctypes.byref(dwm.dwm_rms_info_t())) == BAD
    assert L.dwm_matmul_plan_info(None, ctypes.byref(dwm.dwm_matmul_info_t())) == BAD
    assert L.dwm_rms_set_variant(None, b"forward", 0) == BAD and L.dwm_matmul_set_variant(None, b"kernel", 0) == BAD
    assert L.dwm_rms_forward(None, ONE, None, None, None, ONE, None, None, None, None) == BAD
    assert L.dwm_rms_backward(None, ONE, None, ONE, None, None, ONE, ONE, None, None) == BAD
    assert L.dwm_act_forward(None, ONE, None, ONE, None, None) == BAD
    assert L.dwm_act_backward(None, ONE, ONE, None, None, ONE, None, None) == BAD
    assert L.dwm_matmul(None, ONE, ONE, None, None, ONE, None, None, None) == BAD
    assert L.dwm_matmul_packed(None, P(ONE, ONE), P(ONE, ONE), None, None, ONE, None, None, None) == BAD


def test_rms_calls_that_are_refused(rms):
    f, b, ok = dwm.dwm_rms_forward, dwm.dwm_rms_backward, P(ONE, ONE)
    for args in ((None, None, None, None, ONE), (ONE, None, None, ONE, ONE),  # no x; z without a residual
                 (ONE, ONE, None, None, None), (ONE + 1, None, None, None, ONE), (ONE, ONE + 1, None, None, ONE), (ONE, None, ONE + 2, None, ONE),
                 (ONE, ONE, None, ONE + 1, ONE), (ONE, None, None, None, ONE + 1), (ONE, None, None, None, ONE, P(ONE, None)), (ONE, None, None, None, ONE, P(ONE + 8, ONE)),
                 (ONE, None, None, None, ONE, None, P(ONE, ONE + 1)), (ONE, None, None, None, ONE, None, None, ONE + 2)):
        _refused(BAD, f, rms, *args)
    for args in ((None, None, ONE, None, None, ONE, ONE, None), (ONE, None, None, None, None, ONE, ONE, None), (ONE, None, ONE, ok, None, ONE, ONE, None),
                 (ONE, None, ONE, None, None, None, ONE, None), (ONE, None, ONE, None, None, ONE, None, None), (ONE + 1, None, ONE, None, None, ONE, ONE, None),
                 (ONE, ONE + 1, ONE, None, None, ONE, ONE, None), (ONE, None, ONE + 1, None, None, ONE, ONE, None), (ONE, None, ONE, None, ONE + 2, ONE, ONE, None),
                 (ONE, None, ONE, None, None, ONE + 2, ONE, None), (ONE, None, ONE, None, None, ONE, ONE + 1, None), (ONE, None, ONE, None, None, ONE, ONE, ONE + 2),
                 (ONE, None, None, P(None, ONE), None, ONE, ONE, None)):
        _refused(BAD, b, rms, *args)
    _refused(dwm.DWM_ERR_WORKSPACE, b, rms, ONE, None, ONE, None, None, ONE, ONE, ONE)


def test_rms_plan(rms):
    info = dwm.dwm_rms_plan_info(rms)
    assert (info.rows, info.C) == (4, 96) and dwm.dwm_rms_workspace_bytes(rms) == info.splits * 96 * 4
    for name, stride, status in (("q", 96, BAD), ("x", 95, BAD), ("x", 1 << 39, OUT)):
        _refused(status, dwm.dwm_rms_set_stride, rms, name, stride)
    for stage, v in (("sideways", 0), ("forward", 15), ("forward", 1), ("backward", 15), ("backward", 1)):
        _refused(BAD, dwm.dwm_rms_set_variant, rms, stage, v)
    dwm.dwm_rms_set_variant(rms, "forward", 0)
    assert dwm.dwm_rms_plan_info(rms).forward_kernel == 0
    dwm.dwm_rms_set_variant(rms, "forward", -1)
    assert dwm.dwm_rms_plan_info(rms).forward_kernel == info.forward_kernel
    n = dwm.dwm_rms_workspace_bytes(rms)
    for ws, bytes_ in ((None, n), (ONE + 4, n), (ONE, n - 1)):
        _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_rms_set_workspace, rms, ws, bytes_)
    dwm.dwm_rms_set_workspace(rms, ONE, n)
    _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_rms_set_variant, rms, "backward", 0)
    dwm.dwm_rms_set_variant(rms, "forward", 0)


def test_act_calls_that_are_refused(act):
    f, b, ok = dwm.dwm_act_forward, dwm.dwm_act_backward, P(ONE, ONE)
    for args in ((None, None, ONE), (ONE, None, None), (ONE + 1, None, ONE), (ONE, ONE + 2, ONE), (ONE, None, ONE + 1), (ONE, None, ONE, P(ONE, None))):
        _refused(BAD, f, act, *args)
    for args in ((None, ONE, None, None, ONE, None), (ONE, None, None, None, ONE, None), (ONE, ONE, None, ok, ONE, None), (ONE, None, ONE, ok, ONE, None),
                 (ONE, ONE, None, None, None, None), (ONE + 1, ONE, None, None, ONE, None), (ONE, ONE + 1, None, None, ONE, None), (ONE, ONE, ONE + 2, None, ONE, None),
                 (ONE, ONE, None, None, ONE + 1, None), (ONE, ONE, None, None, ONE, ONE + 2), (ONE, None, ONE, None, ONE, None), (ONE, None, None, P(ONE, ONE + 1), ONE, None)):
        _refused(BAD, b, act, *args)
    _refused(dwm.DWM_ERR_WORKSPACE, b, act, ONE, ONE, None, None, ONE, ONE)
    for name, stride, status in (("z", 96, BAD), ("dy", 95, BAD), ("dx", 1 << 39, OUT)):
        _refused(status, dwm.dwm_act_set_stride, act, name, stride)
    n = dwm.dwm_act_workspace_bytes(act)
    for ws, bytes_ in ((None, n), (ONE + 4, n), (ONE, n - 1)):
        _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_act_set_workspace, act, ws, bytes_)


def test_matmul_calls_that_are_refused():
    plan = dwm.dwm_matmul_plan_create(80, 24, 8, F16, F32, F16, 0, 0)
    packed = dwm.dwm_matmul_plan_create(16, 24, 8, PACKED, BF16, F32, 0, 0)
    ok = P(ONE, ONE)
    try:
        f, g = dwm.dwm_matmul, dwm.dwm_matmul_packed
        for args in ((None, ONE, None, None, ONE), (ONE, None, None, None, ONE), (ONE, ONE, None, None, None), (ONE + 1, ONE, None, None, ONE), (ONE, ONE + 1, None, None, ONE),
                     (ONE, ONE, ONE + 1, None, ONE), (ONE, ONE, None, ONE + 2, ONE), (ONE, ONE, None, None, ONE + 2), (ONE, ONE, None, None, ONE, P(ONE, None)),
                     (ONE, ONE, None, None, ONE, None, P(ONE + 8, ONE))):
            _refused(BAD, f, plan, *args)
        for args in ((None, ok, None, None, ONE), (ok, None, None, None, ONE), (P(ONE, None), ok, None, None, ONE), (ok, P(ONE, ONE + 2), None, None, ONE), (ok, ok, None, None, None),
                     (ok, ok, ONE + 2, None, ONE), (ok, ok, None, ONE + 1, ONE), (ok, ok, None, None, ONE + 1)):
            _refused(BAD, g, packed, *args)
        _refused(BAD, f, packed, ONE, ONE, None, None, ONE)  # each plan has its own call
        _refused(BAD, g, plan, ok, ok, None, None, ONE)
        for p, name, stride, status in ((plan, "a", 7, BAD), (plan, "c", 24, BAD), (plan, "out", 23, BAD), (plan, "b", 1 << 40, OUT), (packed, "a", 8, BAD), (packed, "b", 8, BAD)):
            _refused(status, dwm.dwm_matmul_set_stride, p, name, stride)
        for p, stage, v in ((plan, "kernels", 0), (plan, "kernel", 6), (plan, "kernel", 5), (packed, "kernel", 0), (packed, "kernel", 1), (plan, "splits", 0), (plan, "splits", 65)):
            _refused(BAD, dwm.dwm_matmul_set_variant, p, stage, v)
        assert dwm.dwm_matmul_workspace_bytes(plan) == 0
        dwm.dwm_matmul_set_variant(plan, "splits", 3)
        assert dwm.dwm_matmul_plan_info(plan).splits == 3 and dwm.dwm_matmul_workspace_bytes(plan) == 3 * 80 * 32 * 4
        _refused(dwm.DWM_ERR_WORKSPACE, f, plan, ONE, ONE, None, None, ONE)
        for ws, n in ((None, 1 << 20), (ONE + 4, 1 << 20), (ONE, 3 * 80 * 32 * 4 - 1)):
            _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_matmul_set_workspace, plan, ws, n)
        dwm.dwm_matmul_set_workspace(plan, ONE, 1 << 20)
        _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_matmul_set_variant, plan, "splits", 1)
    finally:
        dwm.dwm_matmul_plan_destroy(plan)
        dwm.dwm_matmul_plan_destroy(packed)


def test_strides_of_operands_across():
    """Across, an operand's rows run along M or N, and there are K of them."""
    plan = dwm.dwm_matmul_plan_create(16, 24, 8, F16, F16, F32, 0, dwm.DWM_A_ACROSS | dwm.DWM_B_ACROSS)
    dwm.dwm_matmul_set_stride(plan, "a", 16)
    dwm.dwm_matmul_set_stride(plan, "b", 24)
    _refused(BAD, dwm.dwm_matmul_set_stride, plan, "a", 15)
    _refused(BAD, dwm.dwm_matmul_set_stride, plan, "b", 23)
    dwm.dwm_matmul_plan_destroy(plan)
