"""Matrix products with their epilogue through the C ABI against 64 bits."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
from branch_gpu import ACT, TYPE, PackedRows, Plan, Rows, n64, normal, param, ptr, stream, within
from test_gpu_rms import packed_within

pytestmark = pytest.mark.gpu


def check(M, N, K, operands="bf16", dtype=None, params="f32", act="none", flags=0, bias=True, residual=True, packed=False, wide=0, off=0, variants=None, inplace=False, seed=3):
    dtype = dtype or ("bf16" if operands == "packed" else operands)
    print("matmul", M, N, K, operands, dtype, params, act, flags, bias, residual, packed, wide, off, variants, flush=True)
    av, bv = normal(M, K, seed), normal(N, K, seed + 1) / np.sqrt(max(K, 1))
    if operands == "packed":
        a, b = PackedRows(M, K, av) if K else None, PackedRows(N, K, bv) if K else None
        a64, b64 = (t.values() if K else np.zeros((n, 0)) for t, n in ((a, M), (b, N)))
    else:
        a = Rows(K, M, operands, wide, off, av.T) if flags & dwm.DWM_A_ACROSS else Rows(M, K, operands, wide, off, av)
        b = Rows(K, N, operands, wide, off, bv.T) if flags & dwm.DWM_B_ACROSS else Rows(N, K, operands, wide, off, bv)
        a64, b64 = a.numpy(), b.numpy()
        a64 = a64.T if flags & dwm.DWM_A_ACROSS else a64
        b64 = b64.T if flags & dwm.DWM_B_ACROSS else b64
    bt = param(N, params, seed + 2) if bias else None
    res = Rows(M, N, dtype, wide, off, normal(M, N, seed + 4)) if residual else None
    r64 = res.numpy() if residual else 0.0
    out = res if inplace else Rows(M, N, dtype, wide, off)
    y8, kept = (PackedRows(M, N), PackedRows(M, N)) if packed else (None, None)
    strides = {"out": out, "residual": res} if operands == "packed" else {"a": a, "b": b, "out": out, "residual": res}
    plan = Plan("matmul", M, N, K, TYPE[operands], TYPE[dtype], TYPE[params], ACT[act], flags, strides=strides, variants=variants)
    try:
        tail = (ptr(bt), ptr(res), out.ptr(), y8.t if packed else None, kept.t if packed else None, stream())
        if operands == "packed":
            dwm.dwm_matmul_packed(plan.plan, a.t if K else None, b.t if K else None, *tail)
        else:
            dwm.dwm_matmul(plan.plan, ptr(a), ptr(b), *tail)
        torch.cuda.synchronize()
        p = a64 @ b64.T + (n64(bt) if bias else 0.0)
        e = ref.matmul_error(a64, b64, operands == "packed") + 2 * ref.U * np.abs(p) + (ref.U * np.abs(n64(bt)) if bias else 0.0)
        v = ref.act(act, p)
        ev = 1.2 * e + ref.act_error(act, p)  # (no slope is over 1.13)
        y = v + r64
        ev = ev + ref.U * np.abs(y)
        within(out.numpy(), y, ev + ref.stored(y, dtype), "out")
        if packed:
            packed_within(kept, p, e, "kept")
            packed_within(y8, y, ev, "out in 8 bits")
        assert out.untouched()
    finally:
        plan.close()
    return out


LAYOUTS = [0, dwm.DWM_A_ACROSS, dwm.DWM_B_ACROSS, dwm.DWM_A_ACROSS | dwm.DWM_B_ACROSS]


@pytest.mark.parametrize("flags", LAYOUTS)
@pytest.mark.parametrize("kernel", range(5))
def test_whole_tiles(kernel, flags):
    for K in (64, 128, 512):
        check(256, 512, K, flags=flags, variants={"kernel": kernel, "splits": 1}, packed=K == 128, act="gelu" if K == 128 else "none")


@pytest.mark.parametrize("flags", LAYOUTS)
@pytest.mark.parametrize("kernel", range(5))
@pytest.mark.parametrize("operands", ["f16", "bf16"])
def test_aligned_odd_tiles(operands, kernel, flags):
    for M, N, K in ((8, 8, 8), (72, 136, 200), (264, 40, 72), (328, 520, 328)):
        check(M, N, K, operands, flags=flags, variants={"kernel": kernel, "splits": 1}, wide=8, packed=True)


@pytest.mark.parametrize("flags", LAYOUTS)
@pytest.mark.parametrize("operands, dtype, params", [("f16", "f16", "f16"), ("f16", "f32", "f16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32")])
def test_any_size(operands, dtype, params, flags):
    for M, N, K in ((1, 1, 1), (3, 5, 7), (65, 33, 129), (130, 257, 77), (200, 100, 1021)):
        check(M, N, K, operands, dtype, params, act="silu", flags=flags, wide=3, off=1, packed=True)


@pytest.mark.parametrize("kernel", [2, 3, 4])
@pytest.mark.parametrize("dtype, params", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_packed_operands(dtype, params, kernel):
    for M, N, K in ((1, 1, 1), (5, 40, 33), (100, 70, 160), (256, 256, 128), (300, 500, 1021)):
        check(M, N, K, "packed", dtype, params, act="gelu", variants={"kernel": kernel, "splits": 1}, wide=1, packed=True)


@pytest.mark.parametrize("operands, kernel", [(o, k) for o in ("f16", "bf16", "packed") for k in range(5) if o != "packed" or k > 1])
def test_parts_of_k(operands, kernel):
    for splits in (2, 5, 64):
        check(136, 264, 1000, operands, act="relu", variants={"kernel": kernel, "splits": splits}, packed=True)
    check(40, 24, 5000, operands)  # as planned


@pytest.mark.parametrize("flags", LAYOUTS)
@pytest.mark.parametrize("operands", ["f16", "bf16"])
def test_odd_rows_laid_out_anew(operands, flags):
    """Kernels for aligned operands asked for where rows are of odd lengths: copies in the workspace, in one and in several parts of K."""
    for kernel in (2, 3, 4):
        for M, N, K in ((40, 72, 129), (65, 33, 200), (300, 261, 1021)):
            check(M, N, K, operands, flags=flags, wide=3, off=1, variants={"kernel": kernel, "splits": 1}, packed=True, act="gelu")
        check(136, 131, 1003, operands, flags=flags, variants={"kernel": kernel, "splits": 3})
    check(1030, 1029, 1027, operands, flags=flags, wide=5)  # as planned


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32])
@pytest.mark.parametrize("operands", ["f16", "bf16", "packed"])
def test_few_rows(operands, M):
    for N, K in ((1, 8), (40, 520), (100, 1024), (33, 4000)):
        check(M, N, K, operands, act="gelu", packed=True, wide=8, variants={"kernel": 5})
        check(M, N, K, operands, residual=False, variants={"kernel": 5})
    check(M, 130, 1021, operands, wide=3, off=1)
    check(M, 33, 1021, operands, wide=3, off=1, packed=True, variants={"kernel": 5})
    check(M, 64, 0, operands, variants={"kernel": 5})
    check(M, 16400, 72, operands, variants={"kernel": 5})


@pytest.mark.parametrize("act", ref.ACTS)
def test_activations(act):
    for operands in ("f16", "packed"):
        check(70, 200, 300, operands, act=act, packed=True)
        check(70, 200, 304, operands, act=act, bias=False, residual=False)


@pytest.mark.parametrize("operands", ["bf16", "packed"])
def test_no_terms_and_no_elements(operands):
    check(20, 40, 0, operands, act="silu", packed=True)
    for M, N in ((0, 8), (8, 0)):
        plan = Plan("matmul", M, N, 16, TYPE[operands], dwm.DWM_BF16, dwm.DWM_F32, 0, 0)
        (dwm.dwm_matmul_packed if operands == "packed" else dwm.dwm_matmul)(plan.plan, None, None, None, None, None, None, None, stream())
        plan.close()


def test_sums_in_place():
    check(100, 200, 300, "bf16", "f32", flags=3, bias=False, inplace=True)
    check(100, 200, 3000, "f16", flags=1, bias=False, inplace=True, variants={"splits": 4})


def test_no_value_of_another_row_gets_in():
    """NaN in the rows and terms around the operands, and in one row of a: it spoils that row alone."""
    for M, N, K in ((70, 90, 100), (20, 90, 100), (3, 40, 72)):
        for operands in ("f16", "bf16"):
            for flags in LAYOUTS:
                for wide in (0, 4, 8, 11):
                    av, bv = normal(M, K, 1), normal(N, K, 2)
                    a = Rows(*((K, M) if flags & 1 else (M, K)), operands, wide, 0)
                    b = Rows(*((K, N) if flags & 2 else (N, K)), operands, wide, 0)
                    a.buffer.fill_(float("nan"))
                    b.buffer.fill_(float("nan"))
                    av[1, 3] = np.nan
                    a.view.copy_(torch.from_numpy(av.T if flags & 1 else av))
                    b.view.copy_(torch.from_numpy(bv.T if flags & 2 else bv))
                    out = Rows(M, N, operands)
                    plan = Plan("matmul", M, N, K, TYPE[operands], TYPE[operands], dwm.DWM_F32, 0, flags, strides={"a": a, "b": b})
                    dwm.dwm_matmul(plan.plan, a.ptr(), b.ptr(), None, None, out.ptr(), None, None, stream())
                    torch.cuda.synchronize()
                    bad = np.isnan(out.numpy())
                    assert bad[1].all() and not np.delete(bad, 1, axis=0).any()
                    plan.close()


@pytest.mark.parametrize("kernel, M", [(2, 40), (3, 40), (4, 40), (5, 20)])
def test_codes_of_nan(kernel, M):
    """An infinity or NaN that was packed spoils its own row of the result, as a row of b its own column."""
    N, K = 70, 200
    av, bv = normal(M, K, 1), normal(N, K, 2)
    av[4, 199], bv[60, 0] = np.inf, np.nan
    a, b, out = PackedRows(M, K, av), PackedRows(N, K, bv), Rows(M, N, "bf16")
    plan = Plan("matmul", M, N, K, dwm.DWM_PACKED, dwm.DWM_BF16, dwm.DWM_F32, 0, 0, variants={"kernel": kernel})
    dwm.dwm_matmul_packed(plan.plan, a.t, b.t, None, None, out.ptr(), None, None, stream())
    torch.cuda.synchronize()
    want = np.zeros((M, N), bool)
    want[4], want[:, 60] = True, True
    assert np.array_equal(np.isnan(out.numpy()), want)
    plan.close()


@pytest.mark.parametrize("flags", LAYOUTS)
@pytest.mark.parametrize("kernel", [2, 3, 4])
def test_no_value_of_another_row_gets_into_copies(kernel, flags):
    """The same where operands of odd rows are laid out anew, eagerly and in a graph replayed over a spoilt workspace."""
    for M, N, K, wide, splits in ((70, 91, 101, 5, 1), (72, 88, 101, 8, 1), (71, 96, 328, 8, 1), (300, 261, 1021, 3, 2)):
        print("matmul copies", M, N, K, wide, splits, flush=True)
        av, bv = normal(M, K, 1), normal(N, K, 2)
        a = Rows(*((K, M) if flags & 1 else (M, K)), "bf16", wide, 0)
        b = Rows(*((K, N) if flags & 2 else (N, K)), "bf16", wide, 0)
        a.buffer.fill_(float("nan"))
        b.buffer.fill_(float("nan"))
        if wide == 8:  # the operand of whole vectors begins at a multiple of sixteen bytes
            a.view, b.view = (t.buffer[:t.rows * t.stride].view(t.rows, t.stride)[:, :t.C] for t in (a, b))
        av[1, 3] = np.nan
        a.view.copy_(torch.from_numpy(av.T if flags & 1 else av))
        b.view.copy_(torch.from_numpy(bv.T if flags & 2 else bv))
        out = Rows(M, N, "bf16")
        plan = Plan("matmul", M, N, K, TYPE["bf16"], TYPE["bf16"], dwm.DWM_F32, 0, flags, strides={"a": a, "b": b}, variants={"kernel": kernel, "splits": splits})
        try:
            def run():
                dwm.dwm_matmul(plan.plan, a.ptr(), b.ptr(), None, None, out.ptr(), None, None, stream())

            run()
            torch.cuda.synchronize()
            first = out.view.clone()
            bad = np.isnan(out.numpy())
            assert bad[1].all() and not np.delete(bad, 1, axis=0).any()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run()
            for _ in range(3):
                plan.ws.fill_(float("nan"))
                out.view.fill_(3.0)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out.view.view(torch.int16), first.view(torch.int16))
        finally:
            plan.close()
