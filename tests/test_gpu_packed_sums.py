"""How far products of packed rows are from 64 bits, by what the matrix cores do with them; sums are seen to the last bits beside a residual that takes off most of them."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import packed_sums as sums
import paper_2002_00552_amd as dwm
from branch_gpu import PackedRows, Plan, Rows, stream, within

pytestmark = pytest.mark.gpu


def packed(v):
    """Into 8 bits on the GPU."""
    x, p = Rows(*v.shape, "f32", values=v.astype(np.float32)), PackedRows(*v.shape)
    dwm.dwm_pack(dwm.DWM_F32, *v.shape, x.ptr(), x.stride, p.t, stream())
    torch.cuda.synchronize()
    return p


def check(a, b, K, variants, low=0.0):
    """`low`: how far, of the whole, the sums have to be below those of the whole products on the average."""
    M, N = a.rows, b.rows
    left, whole, cut, binary32 = sums.product(*(sums.operand(*p.numpy(), K) for p in (a, b)))
    assert (np.abs(left - whole) <= cut).all() and np.abs(whole).max() < 60000
    res, out = Rows(M, N, "f16", values=-whole), Rows(M, N, "f16")
    plan = Plan("matmul", M, N, K, dwm.DWM_PACKED, dwm.DWM_F16, dwm.DWM_F32, 0, 0, variants=variants)
    dwm.dwm_matmul_packed(plan.plan, a.t, b.t, None, res.ptr(), out.ptr(), None, None, stream())
    torch.cuda.synchronize()
    plan.close()
    # out = p + residual, exact in binary32 where the two are within a factor of two, a rounding of p or so where not, and rounded to binary16.
    got = out.numpy() - res.numpy()
    seen = ref.stored(out.numpy(), "f16") + ref.U * np.abs(whole)
    within(got, left, binary32 + seen, "sums of what is left")
    within(got, whole, cut + binary32 + seen, "sums")
    if low:
        assert ((whole - got) / whole).mean() > low


KERNELS = [{"kernel": 2, "splits": 1}, {"kernel": 3, "splits": 1}, {"kernel": 4, "splits": 1}, {"kernel": 2, "splits": 3}, {"kernel": 5}]


def values(M, K, kind, seed):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((M, K))
    if kind != "normal":
        v = np.abs(v)
    if kind == "wide":
        v = v * np.exp(2 * rng.standard_normal((M, K))) / 8  # (sums below the largest binary16)
    return v


@pytest.mark.parametrize("variants", KERNELS)
@pytest.mark.parametrize("kind", ["normal", "positive", "wide"])
@pytest.mark.parametrize("K", [32, 128, 200, 1024, 16384])
def test_sums(K, kind, variants):
    M, N = 20, 48
    a, b = packed(values(M, K, kind, 1)), packed(values(N, K, "positive" if kind == "wide" else kind, 2))
    check(a, b, K, variants)


@pytest.mark.parametrize("variants", KERNELS)
def test_small_products_beside_a_large_one(variants):
    """A product of 1 and, among its seven neighbours and further on, ones of 2^-13, 1.75 * 2^-13 and a little under 2^-13: kept, cut, lost; whole in the next eight."""
    K, M, N = 256, 16, 16
    a, b = PackedRows(M, K), PackedRows(N, K)
    small = [(2.0 ** -7, 2.0 ** -6), (1.75 * 2.0 ** -7, 2.0 ** -6), (1.75 * 2.0 ** -7, 2.0 ** -7)]
    code = {v: i for i, v in enumerate(ref.TABLE[:127])}
    ca, cb = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    for i in range(0, K, 16):
        x, y = small[i // 16 % 3]
        ca[:, i + 1:i + 16], cb[:, i + 1:i + 16] = code[x], code[y]
        ca[:, i], cb[:, i] = code[1.0], code[1.0]
    for p, c in ((a, ca), (b, cb)):
        p.c[:p.nc] = torch.from_numpy(c.reshape(-1)).cuda()
        p.s[:p.ns] = 127
    left, whole, _, _ = sums.product(*(sums.operand(*p.numpy(), K) for p in (a, b)))
    lost = sum(7 * (x * y - np.trunc(x * y * 2.0 ** 13) * 2.0 ** -13) for i in range(0, K, 16) for x, y in [small[i // 16 % 3]])
    assert np.allclose(whole - left, lost, rtol=1e-12) and lost > 0
    check(a, b, K, variants, low=0.5 * lost / whole[0, 0])
