"""The whole-tensor definitions against the ones that go element by element.  No GPU is needed."""
import numpy as np

import branch_reference as ref
import rows_exact as exact


def test_codes_and_scales():
    rng = np.random.default_rng(1)
    for C in (1, 32, 33, 200):
        v = (rng.standard_normal((40, C)) * np.exp(3 * rng.standard_normal((40, C)))).astype(np.float32)
        v[3], v[4, 0], v[5] = 0.0, 448.0, 2.0 ** -140
        v[6, :8] = [448, 1, 2.0 ** -10, 3 * 2.0 ** -10, 17, 18, 19, -9.5][:C]
        v[7, 0] = 448.00003
        for got, want in zip(exact.pack(v.astype(np.float64)), ref.pack(v)):
            assert np.array_equal(got, want)


def test_norms():
    rng = np.random.default_rng(2)
    z, gamma = rng.standard_normal((7, 100)), rng.standard_normal(100)
    for got, want in zip(exact.norm(z, gamma, 1e-5), ref.rms(z, gamma, 1e-5)):
        assert np.allclose(got, want, rtol=1e-14, atol=0)
