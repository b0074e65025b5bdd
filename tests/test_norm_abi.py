"""What the entry points of layer norm and dropout refuse, and what their plans say; no GPU is needed, nothing is launched."""
import ctypes
import math

import pytest

import paper_2002_00552_amd as dwm

ONE = 4096  # an address no call reads


def _refused(status, fn, *args):
    with pytest.raises(dwm.DwmError) as e:
        fn(*args)
    assert e.value.status == status


@pytest.fixture
def plan():
    p = dwm.dwm_norm_plan_create(4, 96, 49, dwm.DWM_F16, dwm.DWM_F32, 1e-5)
    yield p
    dwm.dwm_norm_plan_destroy(p)


@pytest.mark.parametrize("args, status", [
    ((-1, 8, 1, 0, 0, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 0, 1, 0, 0, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 0, 0, 0, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, 3, 0, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, -1, 0, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, dwm.DWM_F16, dwm.DWM_BF16, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, dwm.DWM_F32, dwm.DWM_F16, 1e-5), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, 0, 0, -1e-9), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, 0, 0, math.nan), dwm.DWM_ERR_INVALID_ARG),
    ((1, 8, 1, 0, 0, math.inf), dwm.DWM_ERR_INVALID_ARG),
    ((1, (1 << 20) + 1, 1, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED),
    ((1 << 40, 2, 1, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED),
    ((1, 2, 1 << 40, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED),
    (((1 << 63) - 1, 1 << 20, (1 << 63) - 1, 0, 0, 1e-5), dwm.DWM_ERR_UNSUPPORTED),
])
def test_plans_that_are_refused(args, status):
    _refused(status, dwm.dwm_norm_plan_create, *args)


def test_null_plans_are_refused():
    L = dwm.lib()
    assert L.dwm_norm_plan_create(None, 1, 1, 1, 0, 0, 1e-5) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_plan_destroy(None) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_plan_info(None, ctypes.byref(dwm.dwm_norm_info_t())) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_workspace_bytes(None) == 0
    assert L.dwm_norm_set_workspace(None, ONE, 1 << 20) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_set_stride(None, b"x", 1) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_forward(None, ONE, ONE, ONE, ONE, ONE, ONE, None) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_backward(None, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_join_forward(None, None, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == dwm.DWM_ERR_INVALID_ARG
    assert L.dwm_norm_join_backward(None, None, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == dwm.DWM_ERR_INVALID_ARG


def test_info_and_workspace(plan):
    info = dwm.dwm_norm_plan_info(plan)
    assert (info.outer, info.C, info.inner) == (4, 96, 49)
    assert info.splits >= 1
    need = dwm.dwm_norm_workspace_bytes(plan)
    assert need >= info.splits * 2 * 96 * 4
    _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_set_workspace, plan, None, need)
    _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_set_workspace, plan, ONE + 4, need)
    _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_set_workspace, plan, ONE, need - 1)
    dwm.dwm_norm_set_workspace(plan, ONE, need)


def test_strides(plan):
    for name in ("x", "residual", "z", "y", "dy", "dz", "dx", "dresidual"):
        dwm.dwm_norm_set_stride(plan, name, 96 * 49)
        dwm.dwm_norm_set_stride(plan, name, 96 * 49 + 1)
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_set_stride, plan, name, 96 * 49 - 1)
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_set_stride, plan, name, -96 * 49)
        _refused(dwm.DWM_ERR_UNSUPPORTED, dwm.dwm_norm_set_stride, plan, name, 1 << 62)
    _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_set_stride, plan, "gamma", 96 * 49)
    assert dwm.lib().dwm_norm_set_stride(plan, None, 96 * 49) == dwm.DWM_ERR_INVALID_ARG


def _each_missing(fn, good, required):
    for k in required:
        args = list(good)
        args[k] = None
        _refused(dwm.DWM_ERR_INVALID_ARG, fn, *args)


def _each_misaligned(fn, good, where, by):
    for k in where:
        args = list(good)
        args[k] = ONE + by
        _refused(dwm.DWM_ERR_INVALID_ARG, fn, *args)


def test_calls_that_are_refused(plan):
    forward = [plan] + [ONE] * 6
    _each_missing(dwm.dwm_norm_forward, forward, (1, 4))
    _each_misaligned(dwm.dwm_norm_forward, forward, (1, 4), 1)   # binary16 tensors
    _each_misaligned(dwm.dwm_norm_forward, forward, (2, 3, 5, 6), 2)  # binary32 parameters and statistics
    backward = [plan] + [ONE] * 8
    _each_missing(dwm.dwm_norm_backward, backward, (1, 2, 4, 5))
    _each_misaligned(dwm.dwm_norm_backward, backward, (1, 2, 6), 1)
    _each_misaligned(dwm.dwm_norm_backward, backward, (3, 4, 5, 7, 8), 2)
    _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_backward, plan, ONE, ONE, ONE, ONE, ONE, None, None, None)
    join = [plan, None] + [ONE] * 8
    _each_missing(dwm.dwm_norm_join_forward, join, (2, 3, 6, 7))
    _each_misaligned(dwm.dwm_norm_join_forward, join, (2, 3, 6, 7), 1)
    _each_misaligned(dwm.dwm_norm_join_forward, join, (4, 5, 8, 9), 2)
    back = [plan, None] + [ONE] * 10
    _each_missing(dwm.dwm_norm_join_backward, back, (2, 4, 6, 7))
    _each_misaligned(dwm.dwm_norm_join_backward, back, (2, 3, 4, 8, 9), 1)
    _each_misaligned(dwm.dwm_norm_join_backward, back, (5, 6, 7, 10, 11), 2)
    _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_join_backward, plan, None, ONE, ONE, ONE, ONE, ONE, ONE, None, None, None, None)
    for p, sequence_dev in ((-1e-9, None), (1.0 + 1e-9, None), (math.nan, None), (math.inf, None), (0.5, ONE + 4)):
        drop = dwm.dwm_dropout_t(p, 1, 2, sequence_dev)
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_join_forward, plan, drop, *join[2:])
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_join_backward, plan, drop, *back[2:])
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_dropout_forward, drop, dwm.DWM_F32, 4, ONE, ONE)
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_dropout_backward, drop, dwm.DWM_F32, 4, ONE, ONE)


def test_parameter_gradients_need_the_workspace(plan):
    for dgamma, dbeta in ((ONE, None), (None, ONE)):
        _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_backward, plan, ONE, ONE, ONE, ONE, ONE, ONE, dgamma, dbeta)
        _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_join_backward, plan, None, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, dgamma, dbeta)


def test_dropouts_that_are_refused():
    drop = dwm.dwm_dropout_t(0.5, 1, 2, None)
    for args in ((None, 0, 4, ONE, ONE), (drop, 3, 4, ONE, ONE), (drop, 0, -1, ONE, ONE), (drop, 0, 4, None, ONE), (drop, 0, 4, ONE, None),
                 (drop, dwm.DWM_F32, 4, ONE + 2, ONE), (drop, dwm.DWM_BF16, 4, ONE, ONE + 1)):
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_dropout_forward, *args)
        _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_dropout_backward, *args)
    _refused(dwm.DWM_ERR_UNSUPPORTED, dwm.dwm_dropout_forward, drop, dwm.DWM_F32, (1 << 40) + 1, ONE, ONE)
    dwm.dwm_dropout_forward(drop, dwm.DWM_F32, 0, None, None)  # nothing to do


def test_variants_that_do_not_apply():
    rows, maps = dwm.dwm_norm_plan_create(8, 600, 1, dwm.DWM_F32, dwm.DWM_F32, 1e-5), dwm.dwm_norm_plan_create(8, 600, 7, dwm.DWM_BF16, dwm.DWM_F32, 1e-5)
    try:
        for plan, good, bad in ((rows, (0, 8, 13, -1), (1, 4, 14, 100, 204, 99)), (maps, (0, 111, 112, 113, 211, 213, -1), (1, 110, 210, 212, 214, 300, 100))):
            for stage in ("forward", "backward"):
                for v in good:
                    dwm.dwm_norm_set_variant(plan, stage, v)
                for v in bad:
                    _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_set_variant, plan, stage, v)
            _refused(dwm.DWM_ERR_INVALID_ARG, dwm.dwm_norm_set_variant, plan, "both", 0)
            assert dwm.lib().dwm_norm_set_variant(plan, None, 0) == dwm.DWM_ERR_INVALID_ARG
            dwm.dwm_norm_set_workspace(plan, ONE, 1 << 30)
            dwm.dwm_norm_set_variant(plan, "forward", 0)
            _refused(dwm.DWM_ERR_WORKSPACE, dwm.dwm_norm_set_variant, plan, "backward", 0)
        assert dwm.lib().dwm_norm_set_variant(None, b"forward", 0) == dwm.DWM_ERR_INVALID_ARG
    finally:
        dwm.dwm_norm_plan_destroy(rows)
        dwm.dwm_norm_plan_destroy(maps)
