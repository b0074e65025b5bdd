"""The layer norms, dropouts and joins of residual branches that programs on this library have it do, as cases that can be
timed and compared.

A case is one of these on one GPU, on [outer][C] rows (tokens) or on [N][C][H][W] maps (outputs of the convolutions), both as
[outer][C][inner] with the statistics over the C channels:

* "norm": y of a layer norm, as in serving (no statistics kept);
* "norm_train": its forward and backward pass (y, mean, rstd, dx, dgamma, dbeta);
* "dropout_train": dropout and its gradient, the mask drawn from (seed, sequence) both times and never stored (y, dx);
* "join": a branch joined to its residual stream and the next norm, z = residual + x, y = norm(z), as in serving;
* "join_train": the same with dropout on the branch, forward and backward (z, y, mean, rstd, dx, dresidual, dgamma, dbeta).

Element e of a tensor in its dense order takes word e % 4 of the block that Philox-4x32 with ten rounds (Salmon, Moraes, Dror,
Shaw: Parallel random numbers, as easy as 1, 2, 3; SC 2011) makes of the counter (e / 4, sequence) under the key seed, and is
dropped where that word is below p * 2^32; a kept one is multiplied by 1 / (1 - p), in 32 bits.  A norm reads z as it is
stored: the product and the sum rounded to 32 bits each, then to the tensors' type.

Map sizes are those of the layers of dwm_workloads.py and of the convolutions timed beside this file; row sizes are generic.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_M32 = 0xFFFFFFFF


def _case(name, kind, dtype, params, outer, C, inner, p=0.0, wide=0, eps=1e-5):
    """`wide`: channels that x's rows (maps: images) have beside the ones in use, x being a slice of a wider tensor."""
    case = {"kind": kind, "dtype": dtype, "params": params, "outer": outer, "C": C, "inner": inner, "p": p, "wide": wide,
            "eps": eps}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one pooled image's features before a classifier: nothing but launches and latency
        _case("norm_f32_one_row", "norm", "f32", "f32", 1, 384, 1),
        # a prompt's tokens in serving
        _case("norm_bf16_rows", "norm", "bf16", "bf16", 2048, 4096, 1),
        # reduced-precision serving: the outputs of the down-sampling layer
        _case("norm_f16_maps_28", "norm", "f16", "f32", 32, 256, 28 * 28, eps=1e-6),
        # nothing a multiple of anything: odd channels, image and batch, x cut out of concatenated maps
        _case("norm_train_f32_maps_ragged", "norm_train", "f32", "f32", 5, 93, 18 * 15, wide=31),
        # the benchmark's own layer in training: its outputs, channels first
        _case("norm_train_f32_maps_28", "norm_train", "f32", "f32", 32, 256, 28 * 28, eps=1e-6),
        # a training step's tokens in mixed precision, parameters in 32 bits
        _case("norm_train_bf16_rows", "norm_train", "bf16", "f32", 16384, 2048, 1),
        # a small odd activation in mixed precision
        _case("dropout_train_bf16_odd", "dropout_train", "bf16", "f32", 777, 1021, 1, p=0.1),
        # the outputs of the large-stride first layer
        _case("dropout_train_f32_stem", "dropout_train", "f32", "f32", 128, 96, 55 * 55, p=0.5),
        # one token of one request: what every layer of a decoder does twice for each word
        _case("join_bf16_one_token", "join", "bf16", "bf16", 1, 4096, 1),
        # a full batch of single tokens, wide rows
        _case("join_f16_tokens", "join", "f16", "f16", 192, 8192, 1),
        # a residual block of 3x3 convolutions with 128 channels in training
        _case("join_train_f32_maps_28", "join_train", "f32", "f32", 64, 128, 28 * 28, p=0.2, eps=1e-6),
        # a large training step's tokens: the largest case
        _case("join_train_bf16_rows", "join_train", "bf16", "f32", 16384, 4096, 1, p=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Rows of 16 to 16384 channels, 1 to 65536 of them, or 1 to 128 images of 3 to 1024 channels and 1x1 to 128x128
    pixels, in every type, with x now and then a slice of a wider tensor."""
    most = work(listed()[-1])
    while True:
        kind = rng.choice(["norm", "norm_train", "norm_train", "dropout_train", "join", "join_train", "join_train"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        params = rng.choice(["f32", dtype])
        if rng.random() < 0.5:
            outer, C, inner = _log_int(rng, 1, 65536), _log_int(rng, 16, 16384), 1
            if rng.random() < 0.6:
                C = (C + 7) // 8 * 8
        else:
            H = _log_int(rng, 1, 128)
            W = H if rng.random() < 0.6 else max(1, min(128, H + rng.randint(-6, 6)))
            outer, C, inner = _log_int(rng, 1, 128), _log_int(rng, 3, 1024), H * W
        p = rng.choice([0.1, 0.1, 0.2, 0.5, 0.9]) if kind in ("dropout_train", "join_train") else 0.0
        wide = 0 if kind == "dropout_train" or rng.random() < 0.75 else rng.randint(1, 2 * C)
        case = _case(None, kind, dtype, params, outer, C, inner, p, wide, rng.choice([1e-5, 1e-6]))
        w = work(case)
        if w["bytes"] < 3000 or any(w[k] > most[k] for k in w):
            continue
        if outer * (C + wide) * inner > 2 * 16384 * 4096:
            continue
        return case


def _shape(case):
    return case["outer"], case["C"], case["inner"]


def _inputs(case, seed):
    """The case's tensors on the GPU in their storage types: activations whose channels have offsets and scales of their own
    (a few of them large ones), a residual stream some times as large, gradients and parameters."""
    outer, C, inner = _shape(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (int(seed) % 1_000_003) + 54_321)
    dtype, params = _DTYPES[case["dtype"]], _DTYPES[case["params"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    t = {}
    scale = torch.exp(0.4 * normal(1, C, 1))
    scale[:, torch.randint(C, (1 + C // 256,), generator=g, device="cuda")] *= 8
    t["x"] = (normal(outer, C, inner).mul_(scale).add_(0.3 * scale * normal(1, C, 1))).to(dtype)
    if case["wide"]:  # channels before and behind the ones in use belong to somebody else
        both = torch.full((outer, C + case["wide"], inner), 7.0, dtype=dtype, device="cuda")
        lo = case["wide"] // 2
        both[:, lo:lo + C] = t["x"]
        t["x"] = both[:, lo:lo + C]
    t["gamma"], t["beta"] = (1 + 0.2 * normal(C)).to(params), (0.2 * normal(C)).to(params)
    if case["kind"] in ("join", "join_train"):
        t["residual"] = (normal(outer, C, inner).mul_(2 * scale)).to(dtype)
    if case["kind"].endswith("_train"):
        t["dy"] = normal(outer, C, inner).mul_(0.1).to(dtype)
    if case["kind"] == "join_train":
        t["dz"] = normal(outer, C, inner).mul_(0.1).to(dtype)
    words = np.random.default_rng(int(seed) % (1 << 32)).integers(0, 1 << 32, 3)
    t["seed"], t["sequence"] = int(words[0]) << 32 | int(words[1]), int(words[2])
    return t


class _State:
    """A case's tensors, as a program keeps them: inputs, outputs, and the plan with its workspace."""

    def __init__(self, case, seed):
        self.case, self.kind = dict(case), case["kind"]
        self.plan = None
        outer, C, inner = _shape(case)
        for name, value in _inputs(case, seed).items():
            setattr(self, name, value)

        def empty(like, *shape):
            return torch.empty(shape, dtype=like.dtype, device="cuda")

        self.y = empty(self.x, outer, C, inner)
        self.mean, self.rstd = (torch.empty((outer, inner), dtype=torch.float32, device="cuda") for _ in range(2))
        if self.kind.endswith("_train"):
            self.dx = empty(self.x, outer, C, inner)
            self.dgamma, self.dbeta = empty(self.gamma, C), empty(self.gamma, C)
        if self.kind in ("join", "join_train"):
            self.z = empty(self.x, outer, C, inner)
        if self.kind == "join_train":
            self.dresidual = empty(self.x, outer, C, inner)
        if own:
            self._plan()

    def _plan(self):
        import paper_2002_00552_amd as dwm
        self.dwm = dwm
        types = {"f32": dwm.DWM_F32, "f16": dwm.DWM_F16, "bf16": dwm.DWM_BF16}
        self.type = types[self.case["dtype"]]
        self.drop = dwm.dwm_dropout_t(self.case["p"], self.seed, self.sequence, None)
        if self.kind == "dropout_train":
            return
        outer, C, inner = _shape(self.case)
        self.plan = dwm.dwm_norm_plan_create(outer, C, inner, self.type, types[self.case["params"]], self.case["eps"])
        if self.case["wide"]:
            dwm.dwm_norm_set_stride(self.plan, "x", self.x.stride(0))
        if self.kind.endswith("_train"):
            self.ws = torch.empty(max(dwm.dwm_norm_workspace_bytes(self.plan), 256), dtype=torch.uint8, device="cuda")
            dwm.dwm_norm_set_workspace(self.plan, self.ws.data_ptr(), self.ws.numel())

    def __del__(self):
        if self.plan is not None:
            self.dwm.dwm_norm_plan_destroy(self.plan)


def prepare(case, seed):
    return _State(case, seed)


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    dwm, st = s.dwm, torch.cuda.current_stream().cuda_stream
    if s.kind == "dropout_train":
        dwm.dwm_dropout_forward(s.drop, s.type, s.x.numel(), s.x.data_ptr(), s.y.data_ptr(), st)
        dwm.dwm_dropout_backward(s.drop, s.type, s.x.numel(), s.dy.data_ptr(), s.dx.data_ptr(), st)
        return {"y": s.y, "dx": s.dx}
    if s.kind == "norm":
        dwm.dwm_norm_forward(s.plan, s.x.data_ptr(), s.gamma.data_ptr(), s.beta.data_ptr(), s.y.data_ptr(), None, None, st)
        return {"y": s.y}
    if s.kind == "join":
        dwm.dwm_norm_join_forward(s.plan, None, s.x.data_ptr(), s.residual.data_ptr(), s.gamma.data_ptr(), s.beta.data_ptr(),
                                  s.z.data_ptr(), s.y.data_ptr(), None, None, st)
        return {"z": s.z, "y": s.y}
    mean, rstd = s.mean.data_ptr(), s.rstd.data_ptr()
    if s.kind == "norm_train":
        dwm.dwm_norm_forward(s.plan, s.x.data_ptr(), s.gamma.data_ptr(), s.beta.data_ptr(), s.y.data_ptr(), mean, rstd, st)
        dwm.dwm_norm_backward(s.plan, s.dy.data_ptr(), s.x.data_ptr(), s.gamma.data_ptr(), mean, rstd, s.dx.data_ptr(),
                              s.dgamma.data_ptr(), s.dbeta.data_ptr(), st)
        return {"y": s.y, "mean": s.mean, "rstd": s.rstd, "dx": s.dx, "dgamma": s.dgamma, "dbeta": s.dbeta}
    dwm.dwm_norm_join_forward(s.plan, s.drop, s.x.data_ptr(), s.residual.data_ptr(), s.gamma.data_ptr(), s.beta.data_ptr(),
                              s.z.data_ptr(), s.y.data_ptr(), mean, rstd, st)
    dwm.dwm_norm_join_backward(s.plan, s.drop, s.dy.data_ptr(), s.dz.data_ptr(), s.z.data_ptr(), s.gamma.data_ptr(), mean,
                               rstd, s.dx.data_ptr(), s.dresidual.data_ptr(), s.dgamma.data_ptr(), s.dbeta.data_ptr(), st)
    return {"z": s.z, "y": s.y, "mean": s.mean, "rstd": s.rstd, "dx": s.dx, "dresidual": s.dresidual, "dgamma": s.dgamma,
            "dbeta": s.dbeta}


def _kept(shape, p, seed, sequence):
    """True where an element is kept: the generator in torch's 64-bit integers (a product's low 64 bits are all it needs)."""
    n = math.prod(shape)
    block = torch.arange((n + 3) // 4, device="cuda")
    c = [block & _M32, block >> 32, torch.full_like(block, sequence & _M32), torch.full_like(block, sequence >> 32)]
    k0, k1 = seed & _M32, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & _M32) ^ c[1] ^ k0, b & _M32, ((a >> 32) & _M32) ^ c[3] ^ k1, a & _M32]
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return (torch.stack(c, dim=1).reshape(-1)[:n] >= round(p * 2.0 ** 32)).reshape(shape)


def _dropped(v, kept, p):
    return torch.where(kept, v * (1.0 / (1.0 - p)), 0.0)


def _norm(z, gamma, beta, eps):
    mean = z.mean(dim=1, keepdim=True)
    d = z - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + eps)
    return d * rstd * gamma.float()[:, None] + beta.float()[:, None], mean, rstd


def _norm_backward(dy, z, gamma, mean, rstd):
    xhat = (z - mean) * rstd
    g = dy * gamma.float()[:, None]
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return dx, (dy * xhat).sum(dim=(0, 2)), dy.sum(dim=(0, 2))


def _plain(s):
    """Elementary operations in 32 bits, each output rounded once."""
    dtype, p, eps = s.x.dtype, s.case["p"], s.case["eps"]
    x = s.x.float()
    if s.kind == "dropout_train":
        kept = _kept(x.shape, p, s.seed, s.sequence)
        return {"y": _dropped(x, kept, p).to(dtype), "dx": _dropped(s.dy.float(), kept, p).to(dtype)}
    if s.kind == "norm":
        return {"y": _norm(x, s.gamma, s.beta, eps)[0].to(dtype)}
    if s.kind == "join":
        z = (s.residual.float() + x).to(dtype)
        return {"z": z, "y": _norm(z.float(), s.gamma, s.beta, eps)[0].to(dtype)}
    if s.kind == "norm_train":
        y, mean, rstd = _norm(x, s.gamma, s.beta, eps)
        dx, dgamma, dbeta = _norm_backward(s.dy.float(), x, s.gamma, mean, rstd)
        out = {"dx": dx.to(dtype)}
    else:
        kept = _kept(x.shape, p, s.seed, s.sequence)
        z = (s.residual.float() + _dropped(x, kept, p)).to(dtype)
        y, mean, rstd = _norm(z.float(), s.gamma, s.beta, eps)
        dz, dgamma, dbeta = _norm_backward(s.dy.float(), z.float(), s.gamma, mean, rstd)
        dz = dz + s.dz.float()
        out = {"z": z, "dresidual": dz.to(dtype), "dx": _dropped(dz, kept, p).to(dtype)}
    out.update(y=y.to(dtype), mean=mean[:, 0], rstd=rstd[:, 0], dgamma=dgamma.to(s.gamma.dtype), dbeta=dbeta.to(s.gamma.dtype))
    return out


def work(case):
    """Every input once and every output once; a norm takes some 8 operations an element and its gradient 14, dropout 2."""
    n = math.prod(_shape(case))
    kind, size = case["kind"], {"f32": 4, "f16": 2, "bf16": 2}
    tensors = {"norm": 2, "norm_train": 4, "dropout_train": 4, "join": 3, "join_train": 8}[kind]
    flops = {"norm": 8, "norm_train": 22, "dropout_train": 4, "join": 9, "join_train": 28}[kind]
    vectors = {"norm": 2, "norm_train": 4, "dropout_train": 0, "join": 2, "join_train": 4}[kind]
    stats = 8 * case["outer"] * case["inner"] if kind in ("norm_train", "join_train") else 0
    return {"bytes": tensors * n * size[case["dtype"]] + vectors * case["C"] * size[case["params"]] + stats, "flops": flops * n}


def _kept_exact(shape, p, seed, sequence):
    """The same generator on the host, in numpy's unsigned integers, block by block of the tensor."""
    n, u32 = math.prod(shape), np.uint64(32)
    low, out = np.uint64(_M32), np.empty((n + 3) // 4 * 4, dtype=bool)
    limit = np.uint64(round(p * 2.0 ** 32))
    for at in range(0, (n + 3) // 4, 1 << 18):
        e = np.arange(at, min(at + (1 << 18), (n + 3) // 4), dtype=np.uint64)
        w0, w1 = e & low, e >> u32
        w2, w3 = np.full_like(e, sequence & _M32), np.full_like(e, sequence >> 32)
        for r in range(10):
            key0 = np.uint64((seed + r * 0x9E3779B9) & _M32)
            key1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & _M32)
            p0, p1 = w0 * np.uint64(0xD2511F53), w2 * np.uint64(0xCD9E8D57)
            w0, w1, w2, w3 = (p1 >> u32) ^ w1 ^ key0, p1 & low, (p0 >> u32) ^ w3 ^ key1, p0 & low
        words = out[4 * at:4 * (at + len(e))].reshape(-1, 4)
        for j, w in enumerate((w0, w1, w2, w3)):
            words[:, j] = w >= limit
    return torch.from_numpy(out[:n].reshape(shape)).cuda()


def exact(case, seed):
    """The definitions in 64 bits, from the raw moments and the derivative written out, channels last."""
    t = _inputs(case, seed)
    kind, p, C = case["kind"], case["p"], case["C"]
    dtype = _DTYPES[case["dtype"]]
    keep = _kept_exact(_shape(case), p, t["seed"], t["sequence"]).double() / (1.0 - p) if kind in ("dropout_train", "join_train") else None
    if kind == "dropout_train":
        return {"y": t["x"].double() * keep, "dx": t["dy"].double() * keep}
    out, z = {}, t["x"].double()
    if kind in ("join", "join_train"):
        out["z"] = t["residual"].double() + (z if keep is None else z * keep)
        # what the norm reads: z as it is stored, the product and the sum rounded to 32 bits before it is rounded to its type
        branch = t["x"].float() if keep is None else t["x"].float() * (keep > 0).float() * (1.0 / (1.0 - p))
        z = (t["residual"].float() + branch).to(dtype).double()
    gamma, beta = t["gamma"].double().view(1, 1, C), t["beta"].double().view(1, 1, C)
    z = z.transpose(1, 2).contiguous()
    m1 = z.sum(-1, keepdim=True) / C
    z -= m1
    s2 = (z * z).sum(-1, keepdim=True) / C + case["eps"]
    out["y"] = (z / s2.sqrt() * gamma + beta).transpose(1, 2)
    if kind in ("norm", "join"):
        return out
    out["mean"], out["rstd"] = m1[..., 0], s2[..., 0] ** -0.5
    dy = t["dy"].double().transpose(1, 2).contiguous()
    out["dgamma"], out["dbeta"] = (dy * (z / s2.sqrt())).sum(dim=(0, 1)), dy.sum(dim=(0, 1))
    dy *= gamma
    d = dy / s2.sqrt() - dy.sum(-1, keepdim=True) / (C * s2.sqrt()) - z * ((dy * z).sum(-1, keepdim=True) / (C * s2 ** 1.5))
    d = d.transpose(1, 2)
    if kind == "join_train":
        d = d + t["dz"].double()
        out["dresidual"], out["dx"] = d, d * keep
    else:
        out["dx"] = d
    return out
