"""Root-mean-square norms to the last bit that is stated: one rounding in y and in rstd, y in 8 bits as the exact value has it."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
import rows_exact as exact
from branch_gpu import TYPE, PackedRows, Plan, Rows, ptr, stream, within

pytestmark = pytest.mark.gpu


class Norm:
    """y, y in 8 bits and rstd of rows that are binary32 or of a type that holds them."""

    def __init__(self, z, gamma, eps, dtype="f32", variant=-1):
        rows, C = z.shape
        x, self.y, self.y8, self.rstd = Rows(rows, C, dtype, values=z), Rows(rows, C, dtype), PackedRows(rows, C), torch.empty(rows, device="cuda")
        g = torch.from_numpy(gamma.astype(np.float32)).cuda()
        plan = Plan("rms", rows, C, TYPE[dtype], dwm.DWM_F32, eps, variants={"forward": variant})
        dwm.dwm_rms_forward(plan.plan, x.ptr(), None, ptr(g), None, self.y.ptr(), self.y8.t, None, ptr(self.rstd), stream())
        torch.cuda.synchronize()
        plan.close()
        z64 = x.numpy()
        self.want, self.root = exact.norm(z64, gamma.astype(np.float32).astype(np.float64), eps)

    def check_codes(self):
        codes, scales = self.y8.numpy()
        want = exact.pack(self.want)
        self.y8.check()
        assert np.array_equal(scales, want[1]), "%d scales differ" % (scales != want[1]).sum()
        differ = codes != want[0]
        assert not differ.any(), "%d of %d codes differ, the first at %s" % (differ.sum(), codes.size, np.argwhere(differ)[0])

    def check_values(self, dtype="f32"):
        tolerance = exact.one_rounding(self.want, self.root[:, None])
        within(self.y.numpy(), self.want, tolerance + (0 if dtype == "f32" else ref.stored(self.want, dtype)), "y")
        within(self.rstd.double().cpu().numpy(), self.root, exact.one_rounding(self.root), "rstd")


def rows_on_borders(C, eps, size, ties, seed):
    """A row and a gamma whose y = z rstd gamma lie within a rounding or two of the ties between two codes under the scale byte 127: `ties` are drawn from; in each block of 32 one
    value of 300 (which makes that scale), or, in every fourth block, of some 448 (which decides on the scale itself)."""
    rng = np.random.default_rng(seed)
    z = (size * (0.5 + rng.random((1, C))) * rng.choice([-1, 1], (1, C))).astype(np.float32)
    _, rstd = exact.norm(z.astype(np.float64), 1.0, eps)
    target = rng.choice(ties, C) * rng.choice([-1, 1], C)
    target[::32] = 300.0
    target[::128] = 448.0
    return z, (target / (z[0].astype(np.float64) * rstd[0])).astype(np.float32)


NORMAL = np.array([(8 + m + 0.5) * 2.0 ** (e - 3) for e in range(-6, 8) for m in range(8)])
NORMAL = NORMAL[NORMAL < 220]
SMALL = np.array([(m + 0.5) * 2.0 ** -9 for m in range(8)])  # between the codes below the smallest binade: odd multiples of 2^-10


@pytest.mark.parametrize("variant", [-1, 0])
@pytest.mark.parametrize("ties", [NORMAL, SMALL], ids=["normal", "small"])
def test_codes_at_borders(ties, variant):
    for seed in range(8):
        C = (4096, 1000, 8192, 96)[seed % 4]
        z, gamma = rows_on_borders(C, 1e-6, 1.0, ties, seed)
        norm = Norm(z, gamma, 1e-6, variant=variant)
        near = np.abs(norm.want.astype(np.float32).astype(np.float64) - norm.want) > 0
        assert near.any()
        norm.check_codes()
        norm.check_values()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_codes_of_many_values(dtype):
    """Some 10^7 values, as they come."""
    rng = np.random.default_rng(5)
    rows, C = 2500, 4096
    z = (rng.standard_normal((rows, C)) * np.exp(0.4 * rng.standard_normal(C))).astype(np.float32)
    norm = Norm(z, (1 + 0.2 * rng.standard_normal(C)).astype(np.float32), 1e-5, dtype)
    norm.check_codes()
    norm.check_values(dtype)


@pytest.mark.parametrize("eps", [1e-5, 1e-6, 3e-7, 1e-12])
def test_eps_counts_in_64_bits(eps):
    """Rows far below the root of eps, which rstd then comes from."""
    for seed in range(4):
        z, gamma = rows_on_borders(4096, eps, 1e-3 * np.sqrt(eps), NORMAL, seed)
        norm = Norm(z, gamma, eps)
        norm.check_codes()
        norm.check_values()


@pytest.mark.parametrize("variant", [-1, 0])
@pytest.mark.parametrize("size, by", [(1e-30, 1e-10), (1e-36, 1e-4), (1e30, 1e12), (1e37, 1e5), (1e-12, 1e30), (1e12, 1e-30)])
def test_far_rows_and_far_gammas(size, by, variant):
    """z * gamma leaves binary32, y does not."""
    rng = np.random.default_rng(3)
    z = (size * rng.standard_normal((5, 700))).astype(np.float32)
    norm = Norm(z, (by * (1 + rng.random(700))).astype(np.float32), 0.0, variant=variant)
    norm.check_values()
    norm.check_codes()
