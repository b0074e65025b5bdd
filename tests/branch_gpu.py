"""Helpers of the GPU tests over rows: tensors inside wider buffers, packed rows with guards, plans with workspaces of exact size."""
import numpy as np
import torch

import branch_reference as ref
import paper_2002_00552_amd as dwm

TYPE = {"f32": dwm.DWM_F32, "f16": dwm.DWM_F16, "bf16": dwm.DWM_BF16, "packed": dwm.DWM_PACKED}
ACT = {"none": dwm.DWM_ACT_NONE, "relu": dwm.DWM_ACT_RELU, "gelu": dwm.DWM_ACT_GELU, "silu": dwm.DWM_ACT_SILU}
POISON = 77.0


def stream():
    return torch.cuda.current_stream().cuda_stream


class Rows:
    """[rows][C] inside rows of C + wide that start `off` elements into their buffer."""

    def __init__(self, rows, C, dtype, wide=0, off=0, values=None):
        self.rows, self.C, self.stride = rows, C, C + wide
        self.buffer = torch.full((off + rows * self.stride + 16,), POISON, dtype=ref.TYPES[dtype], device="cuda")
        self.view = self.buffer[off:off + rows * self.stride].view(rows, self.stride)[:, wide // 2:wide // 2 + C]
        if values is not None:
            self.view.copy_(torch.as_tensor(values).to(ref.TYPES[dtype]))

    def ptr(self):
        return self.view.data_ptr()

    def numpy(self):
        return self.view.float().cpu().numpy().astype(np.float64)

    def untouched(self):
        inside = self.view.clone()
        self.view.fill_(POISON)
        ok = bool((self.buffer == POISON).all())
        self.view.copy_(inside)
        return ok


class PackedRows:
    def __init__(self, rows, C, values=None):
        self.rows, self.C = rows, C
        nc, ns = dwm.dwm_packed_codes_bytes(rows, C), dwm.dwm_packed_scales_bytes(rows, C)
        assert nc == rows * 32 * ref.blocks(C) and ns == rows * ((C + 127) // 128 * 4)
        self.c, self.s = (torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda") for n in (nc, ns))
        self.nc, self.ns = nc, ns
        self.t = dwm.dwm_packed_t(self.c.data_ptr(), self.s.data_ptr())
        if values is not None:
            codes, scales = ref.pack(np.asarray(values, np.float32))
            self.c[:nc] = torch.from_numpy(codes.reshape(-1)).cuda()
            self.s[:ns] = torch.from_numpy(scales.reshape(-1)).cuda()

    def numpy(self):
        return (self.c[:self.nc].cpu().numpy().reshape(self.rows, -1), self.s[:self.ns].cpu().numpy().reshape(self.rows, -1))

    def values(self):
        return ref.unpack(*self.numpy(), self.C)

    def check(self):
        """Zeros behind the last channel and block, nothing written behind the whole."""
        codes, scales = self.numpy()
        assert (self.c[self.nc:] == 0xA5).all() and (self.s[self.ns:] == 0xA5).all(), "written behind packed rows"
        assert not codes[:, self.C:].any() and not scales[:, ref.blocks(self.C):].any(), "padding that is not zero"


class Plan:
    """A plan of `family` ("rms", "act", "matmul") with its workspace and a guard behind it."""

    def __init__(self, family, *args, strides=None, variants=None):
        self.family = family
        self.plan = getattr(dwm, "dwm_%s_plan_create" % family)(*args)
        for name, t in (strides or {}).items():
            if t is not None:
                getattr(dwm, "dwm_%s_set_stride" % family)(self.plan, name, t.stride)
        for stage, v in (variants or {}).items():
            getattr(dwm, "dwm_%s_set_variant" % family)(self.plan, stage, v)
        self.n = getattr(dwm, "dwm_%s_workspace_bytes" % family)(self.plan) // 4
        self.ws = torch.full((self.n + 64,), float("nan"), dtype=torch.float32, device="cuda")
        if self.n:
            getattr(dwm, "dwm_%s_set_workspace" % family)(self.plan, self.ws.data_ptr(), self.n * 4)

    def close(self):
        torch.cuda.synchronize()
        assert bool(torch.isnan(self.ws[self.n:]).all()), "written behind the workspace"
        getattr(dwm, "dwm_%s_plan_destroy" % self.family)(self.plan)


def ptr(t):
    return None if t is None else t.data_ptr() if isinstance(t, torch.Tensor) else t.ptr()


def param(C, dtype, seed, mean=0.0):
    rng = np.random.default_rng(seed)
    return torch.from_numpy((mean + 0.3 * rng.standard_normal(C)).astype(np.float32)).to(ref.TYPES[dtype]).cuda()


def n64(t):
    return t.double().cpu().numpy()


def within(got, want, tolerance, what):
    got, want = np.asarray(got), np.asarray(want)
    tolerance = np.broadcast_to(tolerance, want.shape)
    if not want.size:
        return
    worst = np.abs(got - want) - tolerance
    assert np.isfinite(got).all() and (worst <= 0).all(), "%s: off by %.4g at %s, %.4g allowed (%g for %g)" % (
        what, np.abs(got - want).flat[worst.argmax()], np.unravel_index(worst.argmax(), want.shape), tolerance.flat[worst.argmax()],
        got.flat[worst.argmax()], want.flat[worst.argmax()])


def normal(rows, C, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((rows, C))
    if kind == "spread":  # blocks of very different sizes
        v = v * np.exp(4 * rng.standard_normal((rows, C)))
    elif kind == "outlier":
        v[:, rng.integers(C)] *= 100
    elif kind == "small":
        v = v * 1e-3
    return v.astype(np.float32)
