"""Layer norm, dropout and the join of a residual branch through the C ABI against 64 bits (norm_reference.py), at the sizes,
types, strides and values where they can go wrong.  Masks, z and dropped tensors have to be right bit for bit; the others are held
to what norm_reference.py derives for binary32 sums and one rounding to the storage type."""
import numpy as np
import pytest
import torch

import norm_reference as ref
import paper_2002_00552_amd as dwm

pytestmark = pytest.mark.gpu

TYPE = {"f32": dwm.DWM_F32, "f16": dwm.DWM_F16, "bf16": dwm.DWM_BF16}
POISON = 77.0


class Tensor:
    """[outer][C][inner] inside a wider tensor (`wide` channels more) that starts `off` elements into its buffer."""

    def __init__(self, shape, dtype, wide=0, off=0, values=None):
        outer, C, inner = shape
        self.stride = (C + wide) * inner
        n = outer * self.stride
        self.buffer = torch.full((off + n + 8,), POISON, dtype=ref.TYPES[dtype], device="cuda")
        self.view = self.buffer[off:off + n].view(outer, C + wide, inner)[:, wide // 2:wide // 2 + C]
        self.outside = None
        if values is not None:
            self.view.copy_(values.to(ref.TYPES[dtype]))

    def ptr(self):
        return self.view.data_ptr()

    def numpy(self):
        return self.view.float().cpu().numpy().astype(np.float64)

    def untouched(self):
        """Whether everything around the tensor still holds what it held."""
        inside = self.view.clone()
        self.view.fill_(POISON)
        ok = bool((self.buffer == POISON).all())
        self.view.copy_(inside)
        return ok


def _values(shape, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal(shape)
    if kind == "offset":  # a mean far from zero
        v = v + 300.0
    elif kind == "outlier":
        v[:, rng.integers(shape[1])] *= 100
    elif kind == "constant":
        v = np.broadcast_to(v[:, :1], shape)
    elif kind == "small":
        v = v * 1e-3
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32))


def _params(C, params, seed):
    rng = np.random.default_rng(seed)
    gamma, beta = (torch.from_numpy((a + 0.5 * rng.standard_normal(C)).astype(np.float32)).to(ref.TYPES[params]).cuda() for a in (1.0, 0.0))
    return gamma, beta


def _ptr(t):
    return None if t is None else t.data_ptr()


class Norm:
    """A plan with its workspace, sized exactly and with a guard behind it."""

    def __init__(self, shape, dtype, params, eps, tensors=None):
        self.plan = dwm.dwm_norm_plan_create(shape[0], shape[1], shape[2], TYPE[dtype], TYPE[params], eps)
        for name, t in (tensors or {}).items():
            dwm.dwm_norm_set_stride(self.plan, name, t.stride)
        n = dwm.dwm_norm_workspace_bytes(self.plan) // 4
        self.ws = torch.full((n + 64,), float("nan"), dtype=torch.float32, device="cuda")
        dwm.dwm_norm_set_workspace(self.plan, self.ws.data_ptr(), n * 4)
        self.n = n

    def close(self):
        torch.cuda.synchronize()
        assert bool(torch.isnan(self.ws[self.n:]).all()), "written behind the workspace"
        dwm.dwm_norm_plan_destroy(self.plan)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _within(got, want, tolerance, what):
    worst = np.abs(got - want) - tolerance
    assert np.isfinite(got).all() and (worst <= 0).all(), "%s: off by %.3g, %.3g allowed" % (
        what, np.abs(got - want).flat[worst.argmax()], np.broadcast_to(tolerance, want.shape).flat[worst.argmax()])


def check(shape, dtype, params, join=False, p=None, eps=1e-5, wide=0, off=0, kind="normal", with_dz=True, seed=3):
    print("norm", shape, dtype, params, "join" if join else "plain", p, wide, off, kind, flush=True)
    outer, C, inner = shape
    n = outer * inner
    names = ["x", "y", "dy", "dx"] + (["residual", "z", "dz", "dresidual"] if join else [])
    t = {name: Tensor(shape, dtype, wide, off + (k % 3 if off else 0),
                      _values(shape, seed + k, kind if name in ("x", "residual") else "normal") if name in ("x", "dy", "residual", "dz") else None)
         for k, name in enumerate(names)}
    gamma, beta = _params(C, params, seed + 20)
    mean, rstd = (torch.full((outer, inner), float("nan"), device="cuda") for _ in range(2))
    dgamma, dbeta = (torch.full_like(gamma, float("nan")) for _ in range(2))
    drop = None if p is None else dwm.dwm_dropout_t(p, 0xABCDEF0123456789, (1 << 33) + 5, None)
    norm = Norm(shape, dtype, params, eps, t)
    try:
        if join:
            dwm.dwm_norm_join_forward(norm.plan, drop, t["x"].ptr(), t["residual"].ptr(), _ptr(gamma), _ptr(beta), t["z"].ptr(), t["y"].ptr(),
                                      _ptr(mean), _ptr(rstd), _stream())
        else:
            dwm.dwm_norm_forward(norm.plan, t["x"].ptr(), _ptr(gamma), _ptr(beta), t["y"].ptr(), _ptr(mean), _ptr(rstd), _stream())
        g64, b64 = gamma.double().cpu().numpy(), beta.double().cpu().numpy()
        if join:
            keep = np.ones(shape, bool) if p is None else ref.kept(shape, p, drop.seed, drop.sequence)
            branch = ref.dropout32(t["x"].numpy().astype(np.float32), keep, p or 0.0)
            want = ref.rounded(t["residual"].numpy().astype(np.float32) + branch, dtype)
            assert torch.equal(t["z"].view.cpu(), want), "z"
        z = t["z" if join else "x"].numpy()
        y, m, r = ref.norm(z, g64, b64, eps)
        t_y, t_mean, t_rstd = ref.tolerances_forward(z, g64, b64, eps, dtype)
        got_m, got_r = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
        _within(t["y"].numpy(), y, t_y, "y")
        _within(got_m, m, t_mean, "mean")
        _within(got_r, r, t_rstd, "rstd")
        if join:
            dwm.dwm_norm_join_backward(norm.plan, drop, t["dy"].ptr(), t["dz"].ptr() if with_dz else None, t["z"].ptr(), _ptr(gamma), _ptr(mean),
                                       _ptr(rstd), t["dx"].ptr(), t["dresidual"].ptr(), _ptr(dgamma), _ptr(dbeta), _stream())
        else:
            dwm.dwm_norm_backward(norm.plan, t["dy"].ptr(), t["x"].ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd), t["dx"].ptr(), _ptr(dgamma),
                                  _ptr(dbeta), _stream())
        dy = t["dy"].numpy()
        dx, dg, db = ref.norm_backward(dy, z, g64, got_m, got_r)
        dz = t["dz"].numpy() if join and with_dz else np.zeros(shape)
        dx = dx + dz
        t_dx, t_dgamma, t_dbeta = ref.tolerances_backward(dy, z, g64, got_m, got_r, dz, dx, dtype, params, dg, db)
        _within(t["dresidual" if join else "dx"].numpy(), dx, t_dx, "dresidual" if join else "dx")
        if join:
            s = float(ref.scale(p or 0.0))
            _within(t["dx"].numpy(), np.where(keep, dx * s, 0.0), np.where(keep, t_dx * s * 1.01 + ref.TINY[dtype], 0.0), "dx")
        _within(dgamma.double().cpu().numpy(), dg, t_dgamma, "dgamma")
        _within(dbeta.double().cpu().numpy(), db, t_dbeta, "dbeta")
        for name in names:
            assert t[name].untouched(), name
        assert n == 0 or bool(torch.isfinite(mean).all())
    finally:
        norm.close()


ROWS = [(1, 1, 1), (3, 2, 1), (1, 7, 1), (5, 8, 1), (2, 9, 1), (70, 16, 1), (33, 31, 1), (9, 64, 1), (300, 65, 1), (17, 129, 1), (64, 256, 1),
        (3, 500, 1), (130, 512, 1), (7, 777, 1), (20, 1024, 1), (11, 1021, 1), (600, 1030, 1), (5, 2048, 1), (9, 2050, 1), (6, 4096, 1), (4, 4099, 1), (3, 8192, 1),
        (2, 8200, 1), (1, 16384, 1), (2, 16390, 1), (1, 32768, 1), (2, 33001, 1)]
MAPS = [(1, 3, 2), (2, 5, 3), (3, 17, 4), (1, 64, 7), (2, 33, 8), (5, 16, 9), (1, 128, 16), (3, 100, 25), (2, 48, 49), (4, 256, 49), (2, 96, 81), (1, 384, 196),
        (5, 93, 270), (2, 65, 225), (3, 31, 1000), (1, 512, 64), (1, 1024, 36), (2, 700, 25), (1, 1500, 20), (2, 2100, 9), (1, 4, 3025), (40, 24, 5)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, dtype):
    check(shape, dtype, "f32")


@pytest.mark.parametrize("dtype, p", [("f32", 0.1), ("f16", 0.5), ("bf16", 0.1)])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=lambda s: "x".join(map(str, s)))
def test_join(shape, dtype, p):
    check(shape, dtype, dtype, join=True, p=p)


SOME = [(33, 31, 1), (64, 256, 1), (7, 777, 1), (5, 2048, 1), (6, 4096, 1), (2, 33001, 1), (3, 17, 4), (4, 256, 49), (5, 93, 270), (1, 512, 64), (2, 2100, 9), (40, 24, 5)]


@pytest.mark.parametrize("dtype, params", [("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_parameters_of_the_tensors_type(shape, dtype, params):
    check(shape, dtype, params)


@pytest.mark.parametrize("p", [None, 0.0, 0.9, 1.0])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_join_without_dropout_and_with_much(shape, p):
    check(shape, "f32", "f32", join=True, p=p, with_dz=p != 0.9)
    check(shape, "bf16", "f32", join=True, p=p, with_dz=p != 0.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("join", [False, True])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_slices_and_odd_addresses(shape, join, dtype):
    """Tensors inside wider ones, at every address that is a multiple of an element only; nothing around them is written."""
    check(shape, dtype, "f32", join=join, p=0.3 if join else None, wide=3, off=1)
    check(shape, dtype, "f32", join=join, p=0.3 if join else None, wide=8, off=0)


@pytest.mark.parametrize("kind", ["offset", "outlier", "constant", "small"])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_values_that_cost_precision(shape, kind):
    check(shape, "f32", "f32", kind=kind)
    check(shape, "bf16", "f32", join=True, p=0.1, kind=kind)


@pytest.mark.parametrize("shape", [(20000, 24, 1), (3000, 520, 1), (9000, 1500, 1), (64, 40, 900), (30, 260, 784), (300, 70, 49)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_positions(shape):
    check(shape, "f32", "f32")
    check(shape, "f16", "f32", join=True, p=0.2)


@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_what_is_not_asked_for_is_left_out(shape):
    """Missing gamma and beta are ones and zeros; outputs that are not given change nothing of the others."""
    outer, C, inner = shape
    x, dy, dz = (Tensor(shape, "f32", values=_values(shape, k)) for k in (1, 2, 3))
    gamma, beta = _params(C, "f32", 4)
    norm = Norm(shape, "f32", "f32", 1e-5)
    try:
        y, y2 = Tensor(shape, "f32"), Tensor(shape, "f32")
        mean, rstd = (torch.empty((outer, inner), device="cuda") for _ in range(2))
        ones, zeros = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        dwm.dwm_norm_forward(norm.plan, x.ptr(), _ptr(ones), _ptr(zeros), y.ptr(), _ptr(mean), _ptr(rstd), _stream())
        dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, y2.ptr(), None, None, _stream())
        assert torch.equal(y.view, y2.view)
        drop = dwm.dwm_dropout_t(0.25, 1, 2, None)
        full = [Tensor(shape, "f32"), Tensor(shape, "f32"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")]

        def backward(dx, dres, dg, db):
            dwm.dwm_norm_join_backward(norm.plan, drop, dy.ptr(), dz.ptr(), x.ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                       None if dx is None else dx.ptr(), None if dres is None else dres.ptr(), _ptr(dg), _ptr(db), _stream())

        backward(*full)
        for only in range(4):
            part = [Tensor(shape, "f32"), Tensor(shape, "f32"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")]
            backward(*[v if k == only else None for k, v in enumerate(part)])
            a, b = (v.view if only < 2 else v for v in (part[only], full[only]))
            assert torch.equal(a, b), only
    finally:
        norm.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_outputs_in_the_memory_of_their_inputs(shape, dtype):
    outer, C, inner = shape
    x, res, dy, dz = (Tensor(shape, dtype, values=_values(shape, k)) for k in (1, 2, 3, 4))
    y, z, dx, dres = (Tensor(shape, dtype) for _ in range(4))
    gamma, beta = _params(C, "f32", 5)
    mean, rstd = (torch.empty((outer, inner), device="cuda") for _ in range(2))
    grads = [torch.empty(C, device="cuda") for _ in range(4)]
    drop = dwm.dwm_dropout_t(0.2, 9, 9, None)
    norm = Norm(shape, dtype, "f32", 1e-6)
    try:
        def both(x, res, z, y, dy, dz, dx, dres, dg, db):
            dwm.dwm_norm_join_forward(norm.plan, drop, x.ptr(), res.ptr(), _ptr(gamma), _ptr(beta), z.ptr(), y.ptr(), _ptr(mean), _ptr(rstd), _stream())
            dwm.dwm_norm_join_backward(norm.plan, drop, dy.ptr(), dz.ptr(), z.ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd), dx.ptr(), dres.ptr(),
                                       _ptr(dg), _ptr(db), _stream())
        both(x, res, z, y, dy, dz, dx, dres, grads[0], grads[1])
        res2, dy2, dz2, y2 = (Tensor(shape, dtype, values=_values(shape, k)) for k in (2, 3, 4, 4))
        both(x, res2, res2, y2, dy2, dz2, dy2, dz2, grads[2], grads[3])
        for a, b in ((z, res2), (y, y2), (dx, dy2), (dres, dz2)):
            assert torch.equal(a.view, b.view)
        assert torch.equal(grads[0], grads[2]) and torch.equal(grads[1], grads[3])
        # the plain norm: y in x's memory, dx in dy's
        dwm.dwm_norm_forward(norm.plan, x.ptr(), _ptr(gamma), _ptr(beta), y.ptr(), _ptr(mean), _ptr(rstd), _stream())
        x2 = Tensor(shape, dtype, values=_values(shape, 1))
        dwm.dwm_norm_forward(norm.plan, x2.ptr(), _ptr(gamma), _ptr(beta), x2.ptr(), None, None, _stream())
        assert torch.equal(x2.view, y.view)
        dwm.dwm_norm_backward(norm.plan, dy.ptr(), x.ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd), dx.ptr(), _ptr(grads[0]), _ptr(grads[1]), _stream())
        dwm.dwm_norm_backward(norm.plan, dy.ptr(), x.ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd), dy.ptr(), _ptr(grads[2]), _ptr(grads[3]), _stream())
        assert torch.equal(dx.view, dy.view) and torch.equal(grads[0], grads[2]) and torch.equal(grads[1], grads[3])
    finally:
        norm.close()


@pytest.mark.parametrize("value", [float("inf"), float("nan"), -float("inf")])
@pytest.mark.parametrize("shape", SOME, ids=lambda s: "x".join(map(str, s)))
def test_values_that_are_not_finite_stay_in_their_own_norm(shape, value):
    outer, C, inner = shape
    x = Tensor(shape, "f32", values=_values(shape, 1))
    y, want = Tensor(shape, "f32"), Tensor(shape, "f32")
    norm = Norm(shape, "f32", "f32", 1e-5)
    mean, rstd = (torch.zeros((outer, inner), device="cuda") for _ in range(2))
    try:
        dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, want.ptr(), None, None, _stream())
        o, c, i = outer // 2, C - 1, inner // 2
        x.view[o, c, i] = value
        dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, y.ptr(), _ptr(mean), _ptr(rstd), _stream())
        assert bool(torch.isnan(y.view[o, :, i]).all()) and bool(torch.isnan(rstd[o, i])) and not bool(torch.isfinite(mean[o, i]))
        y.view[o, :, i] = want.view[o, :, i]
        assert torch.equal(y.view, want.view)
        # the same place dropped: nothing of it is left
        keep = ref.kept(shape, 0.5, 3, 4)
        gone = [k for k in np.argwhere(~keep)][len(np.argwhere(~keep)) // 2]
        x.view[o, c, i] = 0
        x.view[tuple(gone)] = value
        z, res = Tensor(shape, "f32"), Tensor(shape, "f32", values=_values(shape, 2))
        dwm.dwm_norm_join_forward(norm.plan, dwm.dwm_dropout_t(0.5, 3, 4, None), x.ptr(), res.ptr(), None, None, z.ptr(), y.ptr(), None, None, _stream())
        assert bool(torch.isfinite(z.view).all()) and bool(torch.isfinite(y.view).all())
        assert z.view[tuple(gone)] == res.view[tuple(gone)]
    finally:
        norm.close()


def test_no_rows():
    norm = Norm((0, 12, 5), "bf16", "f32", 1e-5)
    try:
        dgamma, dbeta = (torch.full((12,), float("nan"), device="cuda") for _ in range(2))
        dwm.dwm_norm_forward(norm.plan, None, _ptr(dgamma), None, None, None, None, _stream())
        dwm.dwm_norm_join_forward(norm.plan, None, None, None, None, None, None, None, None, None, _stream())
        dwm.dwm_norm_backward(norm.plan, None, None, None, None, None, None, _ptr(dgamma), _ptr(dbeta), _stream())
        assert bool((dgamma == 0).all()) and bool((dbeta == 0).all())
        dwm.dwm_dropout_forward(dwm.dwm_dropout_t(0.5, 0, 0, None), dwm.DWM_F32, 0, None, None, _stream())
    finally:
        norm.close()


@pytest.mark.parametrize("shape, variant", [((0, 300, 1), v) for v in (0, 5, 8, 10, 12)] + [((0, 40, 30), v) for v in (0, 103, 113, 203)])
def test_no_rows_in_every_kind_of_kernel(shape, variant):
    plan = dwm.dwm_norm_plan_create(*shape, dwm.DWM_F32, dwm.DWM_F32, 1e-5)
    try:
        for stage in ("forward", "backward"):
            if not (variant == 5 and stage == "backward"):  # (a shape of the forward pass alone)
                dwm.dwm_norm_set_variant(plan, stage, variant)
        ws = torch.full((dwm.dwm_norm_workspace_bytes(plan) // 4 + 64,), float("nan"), device="cuda")
        dwm.dwm_norm_set_workspace(plan, ws.data_ptr(), ws.numel() * 4)
        dgamma, dbeta = (torch.full((shape[1],), float("nan"), device="cuda") for _ in range(2))
        dwm.dwm_norm_forward(plan, None, None, None, None, None, None, _stream())
        dwm.dwm_norm_backward(plan, None, None, None, None, None, None, _ptr(dgamma), _ptr(dbeta), _stream())
        assert bool((dgamma == 0).all()) and bool((dbeta == 0).all())
    finally:
        torch.cuda.synchronize()
        dwm.dwm_norm_plan_destroy(plan)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 63, 255, 1023, 1024, 1025, 2047, 2049, 100003])
def test_dropout(n, dtype):
    for p in (0.0, 0.1, 0.5, 0.999, 1.0, 2.0 ** -32, 1e-12, 1 - 1e-12):
        drop = dwm.dwm_dropout_t(p, 2 ** 64 - 3, 2 ** 64 - 1, None)
        x = Tensor((1, n, 1), dtype, off=n % 3, values=_values((1, n, 1), n))
        y = Tensor((1, n, 1), dtype, off=(n + 1) % 3)
        dwm.dwm_dropout_forward(drop, TYPE[dtype], n, x.ptr(), y.ptr(), _stream())
        limit = round(p * 2.0 ** 32)
        keep = (ref.words(n, drop.seed, drop.sequence) >= np.uint64(limit)).reshape(1, n, 1)
        s = np.float32(1.0 / (1.0 - p)) if limit < 2 ** 32 else np.float32(0)
        want = ref.rounded(np.where(keep, x.numpy().astype(np.float32) * s, np.float32(0)), dtype)
        assert torch.equal(y.view.cpu(), want), p
        assert y.untouched()
        dwm.dwm_dropout_backward(drop, TYPE[dtype], n, x.ptr(), x.ptr(), _stream())  # the same mask, in place
        assert torch.equal(x.view, y.view)


def test_dropout_drops_what_is_not_finite():
    n = 4096
    keep = ref.kept((n,), 0.5, 5, 6)
    for value in (float("inf"), float("nan")):
        x = torch.full((n,), value, device="cuda")
        dwm.dwm_dropout_forward(dwm.dwm_dropout_t(0.5, 5, 6, None), dwm.DWM_F32, n, x.data_ptr(), x.data_ptr(), _stream())
        assert torch.equal(x.cpu() == 0, torch.from_numpy(~keep))


def test_sequence_on_the_device_makes_each_replay_of_a_graph_draw_anew():
    """Four replays of a captured training step (join, its gradient, a plain dropout and the counting up of the sequence), with eager
    work and synchronisations in between: each is what eager calls with that sequence give."""
    shape, p, seed = (37, 640, 1), 0.3, 99
    x, res, dy, dz = (Tensor(shape, "bf16", values=_values(shape, k)) for k in (1, 2, 3, 4))
    out = [Tensor(shape, "bf16") for _ in range(5)]
    mean, rstd = (torch.empty(shape[0], device="cuda") for _ in range(2))
    gamma, beta = _params(640, "f32", 5)
    dgamma, dbeta = torch.empty(640, device="cuda"), torch.empty(640, device="cuda")
    counter = torch.full((1,), 7, dtype=torch.int64, device="cuda")
    norm = Norm(shape, "bf16", "f32", 1e-5)

    def step(drop):
        z, y, dx, dres, flat = out
        st = _stream()
        dwm.dwm_norm_join_forward(norm.plan, drop, x.ptr(), res.ptr(), _ptr(gamma), _ptr(beta), z.ptr(), y.ptr(), _ptr(mean), _ptr(rstd), st)
        dwm.dwm_norm_join_backward(norm.plan, drop, dy.ptr(), dz.ptr(), z.ptr(), _ptr(gamma), _ptr(mean), _ptr(rstd), dx.ptr(), dres.ptr(),
                                   _ptr(dgamma), _ptr(dbeta), st)
        dwm.dwm_dropout_forward(drop, dwm.DWM_BF16, 37 * 640, x.ptr(), flat.ptr(), st)
        return [t.view for t in out] + [dgamma, dbeta]

    try:
        captured = dwm.dwm_dropout_t(p, seed, 100, counter.data_ptr())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(captured)
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step(captured)
                counter.add_(1)
        torch.cuda.synchronize()
        previous = None
        for rep in range(4):
            g.replay()
            torch.cuda.synchronize()
            got = [v.clone() for v in [t.view for t in out] + [dgamma, dbeta]]
            want = [v.clone() for v in step(dwm.dwm_dropout_t(p, seed, 100 + 7 + rep, None))]
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b), rep
            assert previous is None or not torch.equal(previous, got[0])
            previous = got[0]
            step(dwm.dwm_dropout_t(0.0, 0, 0, None))  # other values in every buffer before the next replay
            torch.cuda.synchronize()
    finally:
        norm.close()


def test_results_do_not_vary():
    for shape in ((4000, 264, 1), (30, 96, 784)):
        x, dy = (Tensor(shape, "f32", values=_values(shape, k)) for k in (1, 2))
        y, dx = Tensor(shape, "f32"), Tensor(shape, "f32")
        mean, rstd = (torch.empty(shape[0] * shape[2], device="cuda") for _ in range(2))
        C = shape[1]
        norm = Norm(shape, "f32", "f32", 1e-5)
        try:
            first = None
            for _ in range(20):
                dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
                dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, y.ptr(), _ptr(mean), _ptr(rstd), _stream())
                dwm.dwm_norm_backward(norm.plan, dy.ptr(), x.ptr(), None, _ptr(mean), _ptr(rstd), dx.ptr(), _ptr(dgamma), _ptr(dbeta), _stream())
                got = [dgamma, dbeta, dx.view.clone(), y.view.clone()]
                first = first or got
                assert all(torch.equal(a, b) for a, b in zip(first, got))
        finally:
            norm.close()


def test_another_stream_than_the_current_one():
    shape = (64, 512, 1)
    x, y = Tensor(shape, "f32", values=_values(shape, 1)), Tensor(shape, "f32")
    want = Tensor(shape, "f32")
    norm = Norm(shape, "f32", "f32", 1e-5)
    try:
        dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, want.ptr(), None, None, _stream())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        dwm.dwm_norm_forward(norm.plan, x.ptr(), None, None, y.ptr(), None, None, side.cuda_stream)
        side.synchronize()
        assert torch.equal(y.view, want.view)
    finally:
        norm.close()


@pytest.mark.parametrize("shape", [(1 << 20, 2056, 1), (3, 8, 100_000_007)], ids=["rows", "maps"])
def test_offsets_beyond_32_bits(shape):
    """Tensors of more than 2^31 elements (4 GiB of bfloat16): the last positions come out as in a small tensor of their values, and
    the draws of the last elements are those of their places."""
    outer, C, inner = shape
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    x.view(-1)[:].fill_(1.0)
    tail = 4
    part = _values((tail, C, 1), 8) if inner == 1 else _values((1, C, tail), 8)
    where = (slice(outer - tail, outer), slice(None), slice(0, 1)) if inner == 1 else (slice(outer - 1, outer), slice(None), slice(inner - tail, inner))
    x[where] = part.to(torch.bfloat16).cuda()
    y = torch.empty_like(x)
    plan = dwm.dwm_norm_plan_create(outer, C, inner, dwm.DWM_BF16, dwm.DWM_F32, 1e-5)
    try:
        dwm.dwm_norm_forward(plan, x.data_ptr(), None, None, y.data_ptr(), None, None, _stream())
        z = x[where].double().cpu().numpy()
        want = ref.norm(z, np.ones(C), np.zeros(C), 1e-5)[0]
        t_y = ref.tolerances_forward(z, np.ones(C), np.zeros(C), 1e-5, "bf16")[0]
        _within(y[where].double().cpu().numpy(), want, t_y, "y")
        n = x.numel()
        drop = dwm.dwm_dropout_t(0.5, 1, 2, None)
        dwm.dwm_dropout_forward(drop, dwm.DWM_BF16, n, x.data_ptr(), y.data_ptr(), _stream())
        last = 1000
        keep = torch.from_numpy(ref.words(last, 1, 2, n - last) >= np.uint64(1 << 31)).cuda()
        assert torch.equal(y.view(-1)[n - last:], torch.where(keep, x.view(-1)[n - last:] * 2, torch.zeros_like(x.view(-1)[n - last:])))
    finally:
        torch.cuda.synchronize()
        dwm.dwm_norm_plan_destroy(plan)


KERNELS = [*range(0, 14), *range(100, 114), *range(200, 214)]  # dwm_norm_set_variant's numbers


@pytest.mark.parametrize("stage", ["forward", "backward"])
@pytest.mark.parametrize("shape, some", [((70, 40, 1), 4), ((9, 61, 1), 4), ((1500, 1000, 1), 4), ((3, 8190, 1), 2), ((3, 16381, 1), 1), ((6, 32, 49), 12),
                                         ((300, 100, 18), 6), ((2, 700, 270), 3), ((7, 90, 6), 6), ((2, 1999, 5), 2), ((2500, 3, 1), 3)],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_every_kernel(shape, some, stage, monkeypatch):
    """Each kernel that can hold the channels, asked for by number, in training and in a join: at least `some` of them."""
    create = dwm.dwm_norm_plan_create
    for dtype in ("f32", "bf16", "f16"):
        taken = 0
        for variant in KERNELS:
            def asked(*args):
                plan = create(*args)
                dwm.dwm_norm_set_variant(plan, stage, variant)
                info = dwm.dwm_norm_plan_info(plan)
                assert (info.forward_kernel if stage == "forward" else info.backward_kernel) == variant
                return plan

            plan = create(*shape, TYPE[dtype], dwm.DWM_F32, 1e-5)
            try:
                dwm.dwm_norm_set_variant(plan, stage, variant)
            except dwm.DwmError as e:
                assert e.status == dwm.DWM_ERR_INVALID_ARG
                continue
            finally:
                dwm.dwm_norm_plan_destroy(plan)
            taken += 1
            monkeypatch.setattr(dwm, "dwm_norm_plan_create", asked)
            print("kernel", variant, flush=True)
            check(shape, dtype, "f32", kind="offset")
            check(shape, dtype, dtype, join=True, p=0.2, wide=5)
            monkeypatch.undo()
        assert taken > some, taken
