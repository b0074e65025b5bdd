"""The operators over rows together, as a block uses them: a branch in serving with 8-bit operands, one in training with
checkpoints; on other streams, in captured graphs, run again and again, and over tensors of more than 2^31 elements."""
import numpy as np
import pytest
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm
from branch_gpu import ACT, TYPE, PackedRows, Plan, Rows, n64, normal, param, ptr, stream, within
from test_gpu_rms import packed_within

pytestmark = pytest.mark.gpu


class Serving:
    """z = residual + x, n = rms norm of z in 8 bits, h = silu(n w1^T) in 8 bits, out = h w2^T + z."""

    def __init__(self, M, C, F, dtype, seed=1):
        self.M, self.C, self.F, self.dtype = M, C, F, dtype
        self.x, self.residual = (Rows(M, C, dtype, values=normal(M, C, seed + k)) for k in range(2))
        self.gamma = param(C, "f32", seed + 2, 1.0)
        self.w1, self.w2 = PackedRows(F, C, normal(F, C, seed + 3) / np.sqrt(C)), PackedRows(C, F, normal(C, F, seed + 4) / np.sqrt(F))
        self.z, self.out, self.n, self.h = Rows(M, C, dtype), Rows(M, C, dtype), PackedRows(M, C), PackedRows(M, F)
        self.plans = [Plan("rms", M, C, TYPE[dtype], dwm.DWM_F32, 1e-5), Plan("matmul", M, F, C, dwm.DWM_PACKED, TYPE[dtype], dwm.DWM_F32, dwm.DWM_ACT_SILU, 0),
                      Plan("matmul", M, C, F, dwm.DWM_PACKED, TYPE[dtype], dwm.DWM_F32, dwm.DWM_ACT_NONE, 0)]

    def run(self):
        norm, up, down = (p.plan for p in self.plans)
        dwm.dwm_rms_forward(norm, self.x.ptr(), self.residual.ptr(), ptr(self.gamma), self.z.ptr(), None, self.n.t, None, None, stream())
        dwm.dwm_matmul_packed(up, self.n.t, self.w1.t, None, None, None, self.h.t, None, stream())
        dwm.dwm_matmul_packed(down, self.h.t, self.w2.t, None, self.z.ptr(), self.out.ptr(), None, None, stream())

    def check(self):
        """Each operator's outputs from what the one before it stored."""
        z = ref.rounded(self.x.numpy().astype(np.float32) + self.residual.numpy().astype(np.float32), self.dtype)
        assert torch.equal(self.z.view.cpu(), z)
        z = z.double().numpy()
        y, _ = ref.rms(z, n64(self.gamma), 1e-5)
        packed_within(self.n, y, ref.rms_tolerance(z, n64(self.gamma), 1e-5, self.dtype)[0], "the norm")
        n, w1, w2 = self.n.values(), self.w1.values(), self.w2.values()
        p, e = n @ w1.T, ref.matmul_error(n, w1, True)
        packed_within(self.h, ref.act("silu", p), 1.2 * e + ref.act_error("silu", p), "the wide rows")
        h = self.h.values()
        out = h @ w2.T + z
        within(self.out.numpy(), out, ref.matmul_error(h, w2, True) + 3 * ref.U * np.abs(out) + ref.stored(out, self.dtype), "out")

    def outputs(self):
        return [t.clone() for t in (self.z.buffer, self.out.buffer, self.n.c, self.n.s, self.h.c, self.h.s)]

    def close(self):
        for p in self.plans:
            p.close()


@pytest.mark.parametrize("M, C, F, dtype", [(1, 256, 1024, "bf16"), (5, 200, 333, "f16"), (48, 512, 1536, "bf16"), (300, 264, 1000, "f16")])
def test_a_branch_in_serving(M, C, F, dtype):
    s = Serving(M, C, F, dtype)
    s.run()
    torch.cuda.synchronize()
    s.check()
    s.close()


class Training:
    """h = act(x w^T + b) with the sum kept; dp, db from kept; dx = dp w, dw += dp^T x."""

    def __init__(self, M, K, N, dtype, act, seed=5):
        self.M, self.K, self.N, self.dtype, self.act = M, K, N, dtype, act
        self.x, self.w, self.dh = (Rows(r, c, dtype, values=normal(r, c, seed + k) * s) for k, (r, c, s) in enumerate(((M, K, 1.0), (N, K, K ** -0.5), (M, N, 0.1))))
        self.b = param(N, "f32", seed + 7)
        self.h, self.dp, self.dx = Rows(M, N, dtype), Rows(M, N, dtype), Rows(M, K, dtype)
        self.kept = PackedRows(M, N)
        self.start = normal(N, K, seed + 8)
        self.dw, self.db = Rows(N, K, "f32", values=self.start), torch.empty(N, device="cuda")
        t = TYPE[dtype]
        self.plans = [Plan("matmul", M, N, K, t, t, dwm.DWM_F32, ACT[act], 0), Plan("act", ACT[act], M, N, t, dwm.DWM_F32),
                      Plan("matmul", M, K, N, t, t, dwm.DWM_F32, 0, dwm.DWM_B_ACROSS), Plan("matmul", N, K, M, t, dwm.DWM_F32, dwm.DWM_F32, 0, 3)]

    def run(self):
        up, act, data, weights = (p.plan for p in self.plans)
        dwm.dwm_matmul(up, self.x.ptr(), self.w.ptr(), ptr(self.b), None, self.h.ptr(), None, self.kept.t, stream())
        dwm.dwm_act_backward(act, self.dh.ptr(), None, None, self.kept.t, self.dp.ptr(), ptr(self.db), stream())
        dwm.dwm_matmul(data, self.dp.ptr(), self.w.ptr(), None, None, self.dx.ptr(), None, None, stream())
        dwm.dwm_matmul(weights, self.dp.ptr(), self.x.ptr(), None, self.dw.ptr(), self.dw.ptr(), None, None, stream())

    def check(self):
        x, w, dh = self.x.numpy(), self.w.numpy(), self.dh.numpy()
        p = x @ w.T + n64(self.b)
        e = ref.matmul_error(x, w, False) + 3 * ref.U * np.abs(p)
        packed_within(self.kept, p, e, "kept")
        h = ref.act(self.act, p)
        within(self.h.numpy(), h, 1.2 * e + ref.act_error(self.act, p) + ref.stored(h, self.dtype), "h")
        at = self.kept.values()
        g = dh * ref.slope(self.act, at)
        e = np.abs(dh) * ref.slope_error(self.act, at) + 2 * ref.U * np.abs(g)
        within(self.dp.numpy(), g, e + ref.stored(g, self.dtype), "dp")
        within(n64(self.db), g.sum(axis=0), e.sum(axis=0) + ref.rows_error(np.abs(g)) + 2 * ref.U * np.abs(g.sum(axis=0)), "db")
        dp = self.dp.numpy()
        within(self.dx.numpy(), dp @ w, ref.matmul_error(dp, w.T, False) + ref.stored(dp @ w, self.dtype), "dx")
        dw = dp.T @ x + self.start
        within(self.dw.numpy(), dw, ref.matmul_error(dp.T, x.T, False) + 3 * ref.U * np.abs(dw), "dw")

    def close(self):
        for p in self.plans:
            p.close()


@pytest.mark.parametrize("M, K, N, dtype, act", [(1, 64, 128, "bf16", "gelu"), (77, 130, 201, "f16", "silu"), (520, 256, 512, "bf16", "gelu"), (256, 264, 520, "f16", "relu")])
def test_a_product_in_training(M, K, N, dtype, act):
    t = Training(M, K, N, dtype, act)
    t.run()
    torch.cuda.synchronize()
    t.check()
    t.close()


def test_on_another_stream_and_beside_each_other():
    a, b = Serving(33, 320, 640, "bf16", 1), Serving(70, 256, 512, "f16", 30)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in ((a, streams[0]), (b, streams[1])):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s in (a, b):
        s.check()
        s.close()


def test_captured_and_replayed():
    """A graph of a whole branch replayed with new inputs, with eager calls of the same plans between the replays."""
    s, t = Serving(40, 256, 512, "bf16"), Training(136, 128, 264, "bf16", "gelu")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # warm
        s.run()
        t.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
        t.run()
    for k in range(4):
        s.x.view.copy_(torch.from_numpy(normal(40, 256, 50 + k)).to(torch.bfloat16))
        t.x.view.copy_(torch.from_numpy(normal(136, 128, 60 + k)).to(torch.bfloat16))
        t.dw.view.copy_(torch.from_numpy(t.start))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.check()
        t.check()
        got = s.outputs()
        s.run()  # eager, between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, s.outputs()))
    s.close()
    t.close()


def test_results_do_not_vary():
    t = Training(1100, 200, 72, "f16", "silu")
    seen = None
    for _ in range(5):
        t.dw.view.copy_(torch.from_numpy(t.start))
        t.run()
        torch.cuda.synchronize()
        now = [v.clone() for v in (t.h.buffer, t.kept.c, t.dp.buffer, t.dx.buffer, t.dw.buffer, t.db)]
        assert seen is None or all(torch.equal(a, b) for a, b in zip(seen, now))
        seen = now
    t.close()


def test_far_rows_of_norms_activations_and_checkpoints():
    """More than 2^31 elements, by stride and densely: the last rows are right, what lies between rows of a slice is left alone."""
    rows, C, stride = 70000, 96, 40000
    buffer = torch.full((rows * stride,), 3.0, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buffer, (rows, C), (stride, 1), 8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x.copy_(torch.randn(rows, C, generator=g, device="cuda"))
    want = x.clone()
    y, kept = Rows(rows, C, "bf16"), PackedRows(rows, C)
    plan = dwm.dwm_rms_plan_create(rows, C, dwm.DWM_BF16, dwm.DWM_BF16, 1e-5)
    dwm.dwm_rms_set_stride(plan, "x", stride)
    dwm.dwm_rms_forward(plan, x.data_ptr(), None, None, None, y.ptr(), None, kept.t, None, stream())
    torch.cuda.synchronize()
    dwm.dwm_rms_plan_destroy(plan)
    for part in (slice(0, 3), slice(rows - 40, rows)):
        z = want[part].double().cpu().numpy()
        within(y.numpy()[part], ref.rms(z, np.ones(C), 1e-5)[0], ref.rms_tolerance(z, np.ones(C), 1e-5, "bf16")[1], "y")
        codes, scales = (t[part] for t in kept.numpy())
        same = ref.pack(z.astype(np.float32))
        assert np.array_equal(codes, same[0]) and np.array_equal(scales, same[1])
    dwm.dwm_unpack(dwm.DWM_BF16, rows, C, kept.t, x.data_ptr(), stride, stream())  # back into the slice
    torch.cuda.synchronize()
    assert torch.equal(x[-5:].cpu(), torch.from_numpy(ref.unpack(*(t[-5:] for t in kept.numpy()), C)).to(torch.bfloat16))
    x.fill_(3.0)
    assert bool((buffer == 3.0).all())
    del buffer, x
    # dense: 2^31 + some elements of 16 bits through an activation and its gradient
    rows, C = (1 << 31) // 4096 + 3, 4096
    x, y = torch.empty(rows, C, dtype=torch.float16, device="cuda"), torch.empty(rows, C, dtype=torch.float16, device="cuda")
    x.normal_(generator=g)
    codes = torch.empty(dwm.dwm_packed_codes_bytes(rows, C), dtype=torch.uint8, device="cuda")
    scales = torch.empty(dwm.dwm_packed_scales_bytes(rows, C), dtype=torch.uint8, device="cuda")
    packed = dwm.dwm_packed_t(codes.data_ptr(), scales.data_ptr())
    plan = Plan("act", dwm.DWM_ACT_SILU, rows, C, dwm.DWM_F16, dwm.DWM_F32)
    dwm.dwm_act_forward(plan.plan, x.data_ptr(), None, y.data_ptr(), packed, stream())
    p = x[-3:].double().cpu().numpy()
    within(y[-3:].double().cpu().numpy(), ref.act("silu", p), ref.act_error("silu", p) + ref.stored(ref.act("silu", p), "f16"), "y")
    dwm.dwm_act_backward(plan.plan, x.data_ptr(), None, None, packed, y.data_ptr(), None, stream())
    torch.cuda.synchronize()
    same = ref.pack(p.astype(np.float32))
    assert np.array_equal(codes.view(rows, C)[-3:].cpu().numpy(), same[0]) and np.array_equal(scales.view(rows, -1)[-3:].cpu().numpy(), same[1])
    at = ref.unpack(*same, C)
    dx = p * ref.slope("silu", at)
    within(y[-3:].double().cpu().numpy(), dx, np.abs(p) * ref.slope_error("silu", at) + 2 * ref.U * np.abs(dx) + ref.stored(dx, "f16"), "dx")
    plan.close()


@pytest.mark.parametrize("kernel, flags", [(-1, 0), (0, 0), (1, 2), (-1, 1), (-1, 3)])
def test_far_rows_of_products(kernel, flags):
    """Operands and results of more than 2^31 elements: the last rows and columns are right."""
    M, N, K = 70000, 40, 32768
    if flags & 1:
        M, K = K, M
    if flags == 3:
        N = 32
    g = torch.Generator(device="cuda").manual_seed(3)
    a = torch.empty(K if flags & 1 else M, M if flags & 1 else K, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    b = torch.empty(K if flags & 2 else N, N if flags & 2 else K, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = torch.empty(M, N, dtype=torch.float32, device="cuda")
    plan = Plan("matmul", M, N, K, dwm.DWM_BF16, dwm.DWM_F32, dwm.DWM_F32, 0, flags, variants={} if kernel < 0 else {"kernel": kernel})
    dwm.dwm_matmul(plan.plan, a.data_ptr(), b.data_ptr(), None, None, out.data_ptr(), None, None, stream())
    torch.cuda.synchronize()
    a64 = (a[:, -40:].t() if flags & 1 else a[-40:]).double().cpu().numpy()
    b64 = (b.t() if flags & 2 else b).double().cpu().numpy()
    within(out[-40:].double().cpu().numpy(), a64 @ b64.T, ref.matmul_error(a64, b64, False), "out")
    plan.close()


def test_far_results_of_products():
    M, N, K = 70000, 32768, 16
    g = torch.Generator(device="cuda").manual_seed(4)
    a, b = (torch.empty(r, K, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for r in (M, N))
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    codes = torch.empty(dwm.dwm_packed_codes_bytes(M, N), dtype=torch.uint8, device="cuda")
    scales = torch.empty(dwm.dwm_packed_scales_bytes(M, N), dtype=torch.uint8, device="cuda")
    plan = Plan("matmul", M, N, K, dwm.DWM_BF16, dwm.DWM_BF16, dwm.DWM_F32, 0, 0)
    dwm.dwm_matmul(plan.plan, a.data_ptr(), b.data_ptr(), None, None, out.data_ptr(), dwm.dwm_packed_t(codes.data_ptr(), scales.data_ptr()), None, stream())
    torch.cuda.synchronize()
    want = a[-3:].double().cpu().numpy() @ b.double().cpu().numpy().T
    e = ref.matmul_error(a[-3:].double().cpu().numpy(), b.double().cpu().numpy(), False)
    within(out[-3:].double().cpu().numpy(), want, e + ref.stored(want, "bf16"), "out")
    c, s = codes.view(M, N)[-3:].cpu().numpy(), scales.view(M, -1)[-3:].cpu().numpy()
    within(ref.unpack(c, s, N), want, 1.07 * e + ref.half_step(want, s), "out in 8 bits")
    plan.close()
