"""Norms whose mean is far above their deviations, through every kernel: rows and pixels of one value, of one value but for one element, and
of a few neighbouring values, in each storage type, against 64 bits.

What is allowed follows from the kernels' own way, not from the number of channels alone.  With c the longest path of additions that an
element takes (CHAIN), the first mean m0 is off by `first` = c U mean|z| + U max|z| at most.  Deviations from it are exact or off by U
of themselves, and the mean of the deviations puts it right: what is left is a chain over the deviations, 2 c U (mean|z - mean| + first).
The variance is a chain over squares of about var + first^2, of which the square of the correction is taken off again, so rstd is off by
(c + 16) U (1 + (rstd first)^2) of itself.  y has these and its own few roundings; for a row of one value that leaves beta.
"""
import numpy as np
import pytest
import torch

import norm_reference as ref
import paper_2002_00552_amd as dwm

pytestmark = pytest.mark.gpu

TYPE = {"f32": dwm.DWM_F32, "f16": dwm.DWM_F16, "bf16": dwm.DWM_BF16}
KERNELS = [-1, *range(0, 14), *range(100, 114), *range(200, 214)]  # dwm_norm_set_variant's numbers
U = ref.U
# 32 elements of a thread, 6 steps over a wave and 4 over the waves; maps 8, 4 and 16; kernels for any size, at the sizes here: rows 47
# and 8 (12001 channels), maps 47 and 5 (1500 channels, 32 threads a pixel)
CHAIN = 64
EPS = 1e-5


def _tolerances(z, gamma, beta, eps, dtype):
    y, mean, rstd = ref.norm(z, gamma, beta, eps)
    size = np.abs(z)
    first = CHAIN * U * size.mean(axis=1) + U * size.max(axis=1)
    deviation = np.abs(z - mean[:, None])
    t_mean = 2 * CHAIN * U * (deviation.mean(axis=1) + first)
    t_rstd = rstd * (CHAIN + 16) * U * (1 + (rstd * first) ** 2)
    t_y = np.abs(gamma)[:, None] * (rstd * t_mean)[:, None] + np.abs(gamma)[:, None] * deviation * t_rstd[:, None]
    t_y = t_y + 4 * U * (np.abs(y - beta[:, None]) + np.abs(y)) + ref._stored(y, dtype)
    return (y, t_y), (mean, t_mean + 1.01 * U * np.abs(mean)), (rstd, t_rstd)


def _within(got, pair, what):
    want, tolerance = pair
    worst = np.abs(got - want) - tolerance
    at = worst.argmax()
    assert np.isfinite(got).all() and worst.flat[at] <= 0, "%s: off by %.3g, %.3g allowed" % (what, np.abs(got - want).flat[at], tolerance.flat[at])


def _spacing(v, dtype):
    """The distance of neighbours at v."""
    return 2.0 ** np.floor(np.log2(abs(v))) * 2 * ref.ROUNDOFF[dtype]


def _norms(shape, dtype, kind, base, rng):
    """Every norm about a value of its own near base."""
    outer, C, inner = shape
    if kind == "normal":
        return rng.standard_normal(shape)
    if kind == "offset":
        return base + rng.standard_normal(shape)
    v = base * (1 + 0.3 * rng.random((outer, 1, inner)))
    v = ref.rounded(v, dtype).double().numpy()
    step = np.vectorize(_spacing)(v, dtype)
    if kind == "constant":
        return np.broadcast_to(v, shape).copy()
    if kind == "steps":
        return v + step * rng.integers(-3, 4, shape)
    out = np.broadcast_to(v, shape).copy()
    c = rng.integers(C, size=(outer, 1, inner))
    np.put_along_axis(out, c, v + step, axis=1)
    return out


def _kernels(shape, dtype):
    """The kernels that can hold these norms in the forward pass."""
    for variant in KERNELS:
        plan = dwm.dwm_norm_plan_create(*shape, TYPE[dtype], dwm.DWM_F32, EPS)
        try:
            dwm.dwm_norm_set_variant(plan, "forward", variant)
            yield variant, plan
        except dwm.DwmError as e:
            assert e.status == dwm.DWM_ERR_INVALID_ARG
        finally:
            torch.cuda.synchronize()
            dwm.dwm_norm_plan_destroy(plan)


def _stream():
    return torch.cuda.current_stream().cuda_stream


# a plain size, and sizes whose parts of a wave are no powers of two
ROWS = [(5, 56, 1), (5, 112, 1), (4, 224, 1), (3, 448, 1), (4, 500, 1), (4, 512, 1), (3, 1000, 1), (3, 1500, 1), (2, 3000, 1), (2, 12001, 1)]
MAPS = [(2, 56, 50), (1, 96, 49), (2, 224, 33), (2, 300, 50), (1, 500, 40), (1, 512, 49), (1, 1000, 20), (1, 1500, 12)]
BASE = {"f32": (300.1, 12345.678), "f16": (644.0, 3000.0), "bf16": (644.0, 10304.0)}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=lambda s: "x".join(map(str, s)))
def test_means_far_above_the_deviations(shape, dtype):
    outer, C, inner = shape
    rng = np.random.default_rng(17)
    gamma32, beta32 = (1 + 0.5 * rng.standard_normal(C)).astype(np.float32), (0.5 * rng.standard_normal(C)).astype(np.float32)
    gamma, beta = torch.from_numpy(gamma32).cuda(), torch.from_numpy(beta32).cuda()
    cases = []
    for kind, base in [("normal", 0.0), ("offset", BASE[dtype][0])] + [(k, b) for k in ("constant", "one", "steps") for b in BASE[dtype]]:
        x = ref.rounded(_norms(shape, dtype, kind, base, rng), dtype).cuda()
        cases.append(("%s %g" % (kind, base), x, _tolerances(x.double().cpu().numpy(), gamma32.astype(np.float64), beta32.astype(np.float64), EPS, dtype)))
    taken, wrong = 0, []
    for variant, plan in _kernels(shape, dtype):
        taken += 1
        for name, x, (want_y, want_mean, want_rstd) in cases:
            for join in (False, True):
                y, z = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
                mean, rstd = (torch.full((outer, inner), float("nan"), device="cuda") for _ in range(2))
                if join:  # a branch of zeros
                    dwm.dwm_norm_join_forward(plan, None, torch.zeros_like(x).data_ptr(), x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), z.data_ptr(),
                                              y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream())
                else:
                    dwm.dwm_norm_forward(plan, x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream())
                what = "kernel %d, %s, %s" % (variant, name, "join" if join else "norm")
                for out, want, which in ((mean, want_mean, "mean"), (rstd, want_rstd, "rstd"), (y, want_y, "y")):
                    try:
                        _within(out.double().cpu().numpy(), want, which)
                    except AssertionError as e:
                        wrong.append("%s: %s" % (what, str(e).split("\n")[0]))
    assert taken >= 3
    assert not wrong, "%d\n" % len(wrong) + "\n".join(wrong[:12])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 60, 1), (2, 3000, 1), (2, 40, 49), (3, 300, 50), (1, 1024, 36), (1, 1500, 8), (1, 2100, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_norms_of_tiny_values(shape, dtype):
    """Values of 1e-20 and eps = 0, so rstd is 1e20: its square is beyond binary32, the gradient is not.  Bounds of norm_reference.py."""
    outer, C, inner = shape
    rng = np.random.default_rng(23)
    x, dy = (ref.rounded(s * rng.standard_normal(shape), dtype).cuda() for s in (1e-20, 1e-3))
    gamma32 = (1 + 0.5 * rng.standard_normal(C)).astype(np.float32)
    gamma = torch.from_numpy(gamma32).cuda()
    z, dy64, g64 = x.double().cpu().numpy(), dy.double().cpu().numpy(), gamma32.astype(np.float64)
    mean, rstd = (torch.from_numpy(a.astype(np.float32)).cuda() for a in ref.norm(z, g64, np.zeros(C), 0.0)[1:])
    m, r = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    want = ref.norm_backward(dy64, z, g64, m, r)
    allowed = ref.tolerances_backward(dy64, z, g64, m, r, np.zeros(shape), want[0], dtype, "f32", want[1], want[2])
    taken = 0
    for variant in KERNELS:
        plan = dwm.dwm_norm_plan_create(*shape, TYPE[dtype], dwm.DWM_F32, 0.0)
        try:
            dwm.dwm_norm_set_variant(plan, "backward", variant)
            ws = torch.empty(max(dwm.dwm_norm_workspace_bytes(plan), 256), dtype=torch.uint8, device="cuda")
            dwm.dwm_norm_set_workspace(plan, ws.data_ptr(), ws.numel())
            taken += 1
            dx, dgamma, dbeta = torch.full_like(x, float("nan")), torch.full_like(gamma, float("nan")), torch.full_like(gamma, float("nan"))
            args = (gamma.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), _stream())
            dwm.dwm_norm_backward(plan, dy.data_ptr(), x.data_ptr(), *args)
            for got, w, t, name in zip((dx, dgamma, dbeta), want, allowed, ("dx", "dgamma", "dbeta")):
                _within(got.double().cpu().numpy(), (w, t), "kernel %d: %s" % (variant, name))
        except dwm.DwmError as e:
            assert e.status == dwm.DWM_ERR_INVALID_ARG
        finally:
            torch.cuda.synchronize()
            dwm.dwm_norm_plan_destroy(plan)
    assert taken >= 2
