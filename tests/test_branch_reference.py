"""The 64-bit definitions that the kernels over rows are tested against, tested themselves: 8-bit numbers against torch's type,
scales at their borders, gradients against differences.  No GPU is needed."""
import numpy as np
import pytest
import torch

import branch_reference as ref


def test_codes_are_ocp_e4m3():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.TABLE, want, equal_nan=True)


def test_codes_are_the_nearest():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((40, 96)).astype(np.float32) * np.exp(rng.standard_normal((40, 96))).astype(np.float32)
    codes, scales = ref.pack(v)
    by = 2.0 ** (127 - np.repeat(scales[:, :3].astype(np.float64), 32, axis=1))
    want = torch.from_numpy((v * by).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes, want) and not scales[:, 3:].any()
    back = ref.unpack(codes, scales, 96)
    assert (np.abs(back - v) <= ref.half_step(v.astype(np.float64), scales)).all()


@pytest.mark.parametrize("most, s", [(0.0, 0), (448.0, 127), (448.00003, 128), (224.0, 126), (1.0, 119), (1.75, 119), (1.7500001, 120), (3.4e38, 247), (2.0 ** -149, 0)])
def test_scales(most, s):
    assert ref.scale_byte(float(np.float32(most))) == s


@pytest.mark.parametrize("name", ref.ACTS)
def test_slopes_are_derivatives(name):
    p = np.linspace(-9, 9, 1801) + 0.0013
    h = 1e-5
    d = (ref.act(name, p + h) - ref.act(name, p - h)) / (2 * h)
    assert np.abs(d - ref.slope(name, p)).max() < 1e-8


def test_rms_gradient_is_a_derivative():
    rng = np.random.default_rng(2)
    z, dy, gamma, dz = rng.standard_normal((3, 17)), rng.standard_normal((3, 17)), rng.standard_normal(17), rng.standard_normal((3, 17))
    eps, h = 1e-3, 1e-6
    loss = lambda z, g: (ref.rms(z, g, eps)[0] * dy + z * dz).sum()  # noqa: E731
    dx, dgamma = ref.rms_backward(dy, dz, z, gamma, ref.rms(z, gamma, eps)[1])
    for r in range(3):
        for c in range(17):
            e = np.zeros_like(z)
            e[r, c] = h
            assert abs((loss(z + e, gamma) - loss(z - e, gamma)) / (2 * h) - dx[r, c]) < 1e-7
    for c in range(17):
        e = np.zeros(17)
        e[c] = h
        assert abs((loss(z, gamma + e) - loss(z, gamma - e)) / (2 * h) - dgamma[c]) < 1e-7
