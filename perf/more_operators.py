"""The pointwise branch of a residual block as programs on this library have it done, as cases that can be timed and compared:
root-mean-square norms with the residual's addition, activations with their checkpoints in 8 bits, matrix products with an
epilogue, on one GPU, over rows (tokens, pixels with their channels last).

A case is one of these:

* "rms": z = residual + x, y = z * rstd * gamma with rstd = 1 / sqrt(mean of z^2 over the row + eps), as in serving;
* "rms_packed": the same with y in 8 bits, which is then read back;
* "rms_train": the same with z kept in 8 bits and not stored; then dx (with what comes along the residual) and dgamma from it;
* "act_train": y = act(x + bias) with x + bias kept in 8 bits; then dx = dy * act'(kept) and dbias = sum of dx over the rows;
* "keep": a checkpoint alone: rows to 8 bits and back;
* "product": out = act(a b^T + bias) + residual, a [M][K] and b [N][K] both in 16 bits or both in 8;
* "product_train": h = act(x w^T + bias) with the sum before act kept in 8 bits; then dp = dh * act'(kept), dbias, dx = dp w and
  dw = dp^T x;
* "feed": a whole branch in serving with 8-bit operands: z = residual + x, n = rms norm of z in 8 bits, h = silu(n w1^T) in 8 bits,
  out = h w2^T + z.

Rows in 8 bits: each row is cut into blocks of 32 channels, the last one filled up with zeros.  A block has a scale byte s: the
smallest whose 448 * 2^(s - 127) is not below the block's largest finite magnitude (s = 0 for zeros); an element v is the e4m3 code
(four bits of exponent, three of mantissa, no infinities) nearest to v / 2^(s - 127), ties to even.  Codes lie as [rows][32 *
ceil(C / 32)], scales as [rows][4 * ceil(C / 128)].  z is packed as it is stored (rounded to its type), x + bias rounded to 32
bits, the others from 32 bits.

gelu is x * (1 + erf(x / sqrt 2)) / 2, silu x / (1 + exp(-x)).  Sizes are generic, those of the benchmark's own layers (channels,
28 x 28 maps) among them.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_ROWS = ("rms", "rms_packed", "rms_train", "act_train", "keep")


def _case(name, kind, dtype, M, N, K=0, params="f32", act="none", operands="typed", bias=False, residual=False, wide=0, eps=1e-5):
    """Over rows: M rows of N channels.  `wide`: channels that the rows of x (of a product: of a) have beside the ones in use."""
    case = {"kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "params": params, "act": act, "operands": operands, "bias": bias,
            "residual": residual, "wide": wide, "eps": eps}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token of one request: nothing but launches and latency
        _case("rms_bf16_one_token", "rms", "bf16", 1, 4096, params="bf16"),
        # a prompt's rows for products of 8-bit operands
        _case("rms_packed_bf16_rows", "rms_packed", "bf16", 4096, 4096, params="bf16"),
        # nothing a multiple of anything: odd rows and channels, x a slice of wider rows
        _case("rms_train_f16_ragged", "rms_train", "f16", 777, 1021, wide=19, eps=1e-6),
        # a large training step's rows, parameters in 32 bits
        _case("rms_train_bf16_rows", "rms_train", "bf16", 16384, 4096),
        # a small odd activation in training
        _case("act_train_f16_odd", "act_train", "f16", 333, 1003, act="silu", bias=True),
        # the widest activation of a training step
        _case("act_train_bf16_rows", "act_train", "bf16", 16384, 8192, act="gelu", bias=True),
        # the outputs of the benchmark's own layer between its forward and its backward pass: 32 x 256 rows of 28 x 28
        _case("keep_f32_maps_28", "keep", "f32", 32 * 256, 28 * 28),
        # one token of one request: the weights are read once
        _case("product_bf16_one_token", "product", "bf16", 1, 4096, 4096, params="bf16", bias=True, residual=True),
        # odd rows, columns and contraction, a cut out of wider rows
        _case("product_f16_ragged", "product", "f16", 1000, 777, 1021, act="gelu", bias=True, residual=True, wide=7),
        # a batch of single tokens through a whole branch
        _case("feed_bf16_tokens", "feed", "bf16", 48, 4096, 12288, params="bf16", act="silu", operands="packed"),
        # prompts, operands in 8 bits
        _case("product_packed_rows", "product", "bf16", 8192, 8192, 4096, params="bf16", act="silu", operands="packed", bias=True),
        # a training step's first product, forward and backward: the largest case
        _case("product_train_bf16_rows", "product_train", "bf16", 8192, 8192, 2048, params="bf16", act="gelu", bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """1 to 32768 rows of 16 to 16384 channels, products of 1 to 16384 rows and 16 to 16384 columns and terms, in every type, half
    of them of whole vectors and half of any size, now and then out of wider rows."""
    all_work = [work(c) for c in listed()]
    most = {k: max(w[k] for w in all_work) for k in all_work[0]}
    while True:
        kind = rng.choice(["rms", "rms_packed", "rms_train", "rms_train", "act_train", "act_train", "keep", "product", "product",
                           "product", "product_train", "product_train", "feed"])
        rows = kind in _ROWS
        dtype = rng.choice(["f32", "f16", "bf16"] if rows else ["f16", "bf16"])
        params = rng.choice(["f32", dtype]) if kind not in ("product_train", "feed") else dtype
        M, N, K = _log_int(rng, 1, 32768 if rows else 16384), _log_int(rng, 16, 16384), 0 if rows else _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            N, K = (N + 7) // 8 * 8, (K + 7) // 8 * 8
        act = "silu" if kind == "feed" else rng.choice(["relu", "gelu", "silu"] + ["none"] * (kind == "product"))
        operands = "packed" if kind == "feed" or (kind == "product" and rng.random() < 0.4) else "typed"
        bias = kind in ("act_train", "product_train") or (kind == "product" and rng.random() < 0.6)
        residual = kind == "product" and rng.random() < 0.5
        wide = rng.randint(1, 64) if operands == "typed" and kind != "keep" and rng.random() < 0.25 else 0
        case = _case(None, kind, dtype, M, N, K, params, act if not rows or kind == "act_train" else "none", operands, bias, residual,
                     wide, rng.choice([1e-5, 1e-6]))
        w = work(case)
        if w["bytes"] < 3000 or any(w[k] > most[k] for k in w):
            continue
        return case


def _inputs(case, seed):
    """The case's tensors on the GPU in their storage types: activations with a few large channels, a residual stream some times
    as large, gradients, weights and parameters."""
    kind, M, N, K = case["kind"], case["M"], case["N"], case["K"]
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (int(seed) % 1_000_003) + 98_765)
    dtype, params = _DTYPES[case["dtype"]], _DTYPES[case["params"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def activations(rows, C, size=1.0):
        scale = size * torch.exp(0.4 * normal(C))
        scale[torch.randint(C, (1 + C // 256,), generator=g, device="cuda")] *= 8
        return normal(rows, C).mul_(scale)

    def sliced(values):
        if not case["wide"]:
            return values.to(dtype)
        both = torch.full((values.shape[0], values.shape[1] + case["wide"]), 7.0, dtype=dtype, device="cuda")
        lo = case["wide"] // 2
        both[:, lo:lo + values.shape[1]] = values
        return both[:, lo:lo + values.shape[1]]

    t = {}
    if kind in ("rms", "rms_packed", "rms_train"):
        t["x"], t["residual"] = sliced(activations(M, N)), activations(M, N, 2.0).to(dtype)
        t["gamma"] = (1 + 0.2 * normal(N)).to(params)
        if kind == "rms_train":
            t["dy"], t["dz"] = normal(M, N).mul_(0.1).to(dtype), normal(M, N).mul_(0.1).to(dtype)
    elif kind == "act_train":
        t["x"], t["bias"], t["dy"] = sliced(activations(M, N)), (0.3 * normal(N)).to(params), normal(M, N).mul_(0.1).to(dtype)
    elif kind == "keep":
        t["x"] = activations(M, N).to(dtype)
    elif kind == "feed":
        t["x"], t["residual"] = activations(M, N).to(dtype), activations(M, N, 2.0).to(dtype)
        t["gamma"] = (1 + 0.2 * normal(N)).to(params)
        t["w1"], t["w2"] = _pack(normal(K, N) / math.sqrt(N)), _pack(normal(N, K) / math.sqrt(K))
    else:
        a, b = activations(M, K), normal(N, K) / math.sqrt(K)
        t["a"], t["b"] = (_pack(a), _pack(b)) if case["operands"] == "packed" else (sliced(a), b.to(dtype))
        if case["bias"]:
            t["bias"] = (0.3 * normal(N)).to(params)
        if case["residual"]:
            t["residual"] = normal(M, N).mul_(2).to(dtype)
        if kind == "product_train":
            t["dh"] = normal(M, N).mul_(0.1).to(dtype)
    return t


def _two(k):
    """2^k in 32 bits, from -127 to 127, from its pattern."""
    return torch.where(k > -127, (k + 127) << 23, 1 << 22).int().view(torch.float32)


def _pack(v):
    """Values in 32 bits -> (codes, scales), two tensors of bytes."""
    rows, C = v.shape
    blocks = (C + 31) // 32
    v = torch.nn.functional.pad(v, (0, 32 * blocks - C)).view(rows, blocks, 32)
    most = v.abs().amax(dim=2)
    mantissa, exponent = torch.frexp(most)  # most = mantissa * 2^exponent; 448 = 0.875 * 2^9
    s = torch.where(most > 0, (exponent - 9 + (mantissa > 0.875).int() + 127).clamp(min=0), 0)
    codes = (v * _two(127 - s)[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, 32 * blocks)
    return codes, torch.nn.functional.pad(s, (0, -blocks % 4)).to(torch.uint8)


def _unpack(packed, C):
    codes, scales = packed
    rows, blocks = codes.shape[0], codes.shape[1] // 32
    v = codes.view(torch.float8_e4m3fn).float().view(rows, blocks, 32)
    return (v * _two(scales[:, :blocks].int() - 127)[:, :, None]).view(rows, 32 * blocks)[:, :C]


class _State:
    """A case's tensors, as a program keeps them: inputs, outputs, and plans with their workspaces."""

    def __init__(self, case, seed):
        self.case, self.kind = dict(case), case["kind"]
        self.plans = []
        M, N, K = case["M"], case["N"], case["K"]
        dtype, params = _DTYPES[case["dtype"]], _DTYPES[case["params"]]
        self.t = _inputs(case, seed)

        def empty(*shape, dtype=dtype):
            return torch.empty(shape, dtype=dtype, device="cuda")

        def packed(rows, C):
            return (empty(rows, (C + 31) // 32 * 32, dtype=torch.uint8), empty(rows, (C + 127) // 128 * 4, dtype=torch.uint8))

        o = {}
        if self.kind in ("rms", "rms_packed", "feed"):
            o["z"], o["rstd"] = empty(M, N), None
        if self.kind in ("rms", "rms_train", "act_train", "keep", "rms_packed"):
            o["y"] = empty(M, N)
        if self.kind == "rms_packed":
            o["y"] = empty(M, N, dtype=torch.bfloat16)
        if self.kind != "rms" and not self.kind == "product":
            o["kept"] = packed(M, N)
        if self.kind == "rms_train":
            o.update(rstd=empty(M, dtype=torch.float32), dx=empty(M, N), dgamma=empty(N, dtype=params))
        if self.kind == "act_train":
            o.update(dx=empty(M, N), dbias=empty(N, dtype=params))
        if self.kind in ("product", "product_train", "feed"):
            o["out"] = empty(M, N)
        if self.kind == "feed":
            o["h"] = packed(M, K)
        if self.kind == "product_train":
            o.update(dp=empty(M, N), dbias=empty(N, dtype=params), dx=empty(M, K), dw=empty(N, K))
        self.o = o
        if own:
            self._plan()

    def _plan(self):
        import paper_2002_00552_amd as dwm
        self.dwm = dwm
        case, t = self.case, self.t
        M, N, K = case["M"], case["N"], case["K"]
        types = {"f32": dwm.DWM_F32, "f16": dwm.DWM_F16, "bf16": dwm.DWM_BF16}
        type, params = types[case["dtype"]], types[case["params"]]
        act = {"none": dwm.DWM_ACT_NONE, "relu": dwm.DWM_ACT_RELU, "gelu": dwm.DWM_ACT_GELU, "silu": dwm.DWM_ACT_SILU}[case["act"]]
        operands = dwm.DWM_PACKED if case["operands"] == "packed" else type
        self.type = type
        self.ws = []

        def keep(plan, destroy, workspace_bytes, set_workspace):
            self.plans.append((destroy, plan))
            n = workspace_bytes(plan)
            if n:
                self.ws.append(torch.empty(n, dtype=torch.uint8, device="cuda"))
                set_workspace(plan, self.ws[-1].data_ptr(), n)
            return plan

        def rms():
            plan = dwm.dwm_rms_plan_create(M, N, type, params, case["eps"])
            dwm.dwm_rms_set_stride(plan, "x", t["x"].stride(0))
            return keep(plan, dwm.dwm_rms_plan_destroy, dwm.dwm_rms_workspace_bytes, dwm.dwm_rms_set_workspace)

        def activation():
            return keep(dwm.dwm_act_plan_create(act, M, N, type, params), dwm.dwm_act_plan_destroy, dwm.dwm_act_workspace_bytes,
                        dwm.dwm_act_set_workspace)

        def product(M, N, K, act=dwm.DWM_ACT_NONE, flags=0, a=None, b=None):
            plan = dwm.dwm_matmul_plan_create(M, N, K, operands, type, params, act, flags)
            if a is not None:
                dwm.dwm_matmul_set_stride(plan, "a", a.stride(0))
            if b is not None:
                dwm.dwm_matmul_set_stride(plan, "b", b.stride(0))
            return keep(plan, dwm.dwm_matmul_plan_destroy, dwm.dwm_matmul_workspace_bytes, dwm.dwm_matmul_set_workspace)

        if self.kind in ("rms", "rms_packed", "rms_train", "feed"):
            self.rms = rms()
        if self.kind in ("act_train", "product_train"):
            self.act = activation()
        if self.kind == "act_train":
            dwm.dwm_act_set_stride(self.act, "x", t["x"].stride(0))
        if self.kind in ("product", "product_train"):
            self.forward = product(M, N, K, act, a=None if operands == dwm.DWM_PACKED else t["a"])
        if self.kind == "product_train":
            self.data = product(M, K, N, flags=dwm.DWM_B_ACROSS)
            self.weights = product(N, K, M, flags=dwm.DWM_A_ACROSS | dwm.DWM_B_ACROSS, b=t["a"])
        if self.kind == "feed":
            self.up, self.down = product(M, K, N, act), product(M, N, K)
        self.packed = {k: dwm.dwm_packed_t(v[0].data_ptr(), v[1].data_ptr())
                       for k, v in list(t.items()) + list(self.o.items()) if isinstance(v, tuple)}

    def __del__(self):
        for destroy, plan in self.plans:
            destroy(plan)


def prepare(case, seed):
    return _State(case, seed)


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    dwm, st, kind, t, o, packed = s.dwm, torch.cuda.current_stream().cuda_stream, s.kind, s.t, s.o, s.packed
    M, N = s.case["M"], s.case["N"]

    def p(name):
        v = t.get(name, o.get(name))
        return None if v is None else v.data_ptr()

    if kind == "rms":
        dwm.dwm_rms_forward(s.rms, p("x"), p("residual"), p("gamma"), p("z"), p("y"), None, None, None, st)
        return {"z": o["z"], "y": o["y"]}
    if kind == "rms_packed":
        dwm.dwm_rms_forward(s.rms, p("x"), p("residual"), p("gamma"), p("z"), None, packed["kept"], None, None, st)
        dwm.dwm_unpack(dwm.DWM_BF16, M, N, packed["kept"], p("y"), N, st)
        return {"z": o["z"], "y": o["y"]}
    if kind == "rms_train":
        dwm.dwm_rms_forward(s.rms, p("x"), p("residual"), p("gamma"), None, p("y"), None, packed["kept"], p("rstd"), st)
        dwm.dwm_rms_backward(s.rms, p("dy"), p("dz"), None, packed["kept"], p("gamma"), p("rstd"), p("dx"), p("dgamma"), st)
        return {"y": o["y"], "rstd": o["rstd"], "dx": o["dx"], "dgamma": o["dgamma"]}
    if kind == "act_train":
        dwm.dwm_act_forward(s.act, p("x"), p("bias"), p("y"), packed["kept"], st)
        dwm.dwm_act_backward(s.act, p("dy"), None, None, packed["kept"], p("dx"), p("dbias"), st)
        return {"y": o["y"], "dx": o["dx"], "dbias": o["dbias"]}
    if kind == "keep":
        dwm.dwm_pack(s.type, M, N, p("x"), N, packed["kept"], st)
        dwm.dwm_unpack(s.type, M, N, packed["kept"], p("y"), N, st)
        return {"y": o["y"]}
    if kind == "product":
        if s.case["operands"] == "packed":
            dwm.dwm_matmul_packed(s.forward, packed["a"], packed["b"], p("bias"), p("residual"), p("out"), None, None, st)
        else:
            dwm.dwm_matmul(s.forward, p("a"), p("b"), p("bias"), p("residual"), p("out"), None, None, st)
        return {"out": o["out"]}
    if kind == "feed":
        dwm.dwm_rms_forward(s.rms, p("x"), p("residual"), p("gamma"), p("z"), None, packed["kept"], None, None, st)
        dwm.dwm_matmul_packed(s.up, packed["kept"], packed["w1"], None, None, None, packed["h"], None, st)
        dwm.dwm_matmul_packed(s.down, packed["h"], packed["w2"], None, p("z"), p("out"), None, None, st)
        return {"z": o["z"], "out": o["out"]}
    dwm.dwm_matmul(s.forward, p("a"), p("b"), p("bias"), None, p("out"), None, packed["kept"], st)
    dwm.dwm_act_backward(s.act, p("dh"), None, None, packed["kept"], p("dp"), p("dbias"), st)
    dwm.dwm_matmul(s.data, p("dp"), p("b"), None, None, p("dx"), None, None, st)
    dwm.dwm_matmul(s.weights, p("dp"), p("a"), None, None, p("dw"), None, None, st)
    return {"out": o["out"], "dp": o["dp"], "dbias": o["dbias"], "dx": o["dx"], "dw": o["dw"]}


def _act(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v / (1 + torch.exp(-v)) if act == "silu" else v


def _act_gradient(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))
    sigmoid = 1 / (1 + torch.exp(-v))
    return sigmoid * (1 + v * (1 - sigmoid))


def _rms(z, gamma, eps):
    rstd = 1.0 / torch.sqrt((z * z).mean(dim=1, keepdim=True) + eps)
    return z * rstd * gamma.float(), rstd


def _plain(s):
    """Elementary operations in 32 bits, each operator's outputs rounded once."""
    kind, t, case = s.kind, s.t, s.case
    M, N, K, act, dtype = case["M"], case["N"], case["K"], case["act"], _DTYPES[case["dtype"]]
    if kind in ("rms", "rms_packed", "rms_train", "feed"):
        z = (t["residual"].float() + t["x"].float()).to(dtype)
        y, rstd = _rms(z.float(), t["gamma"], case["eps"])
        if kind == "rms":
            return {"z": z, "y": y.to(dtype)}
        if kind == "rms_packed":
            return {"z": z, "y": _unpack(_pack(y), N).to(torch.bfloat16)}
        if kind == "feed":
            h = _act(torch.mm(_unpack(_pack(y), N), _unpack(t["w1"], N).t()), act)
            out = torch.mm(_unpack(_pack(h), K), _unpack(t["w2"], K).t()) + z.float()
            return {"z": z, "out": out.to(dtype)}
        xhat, dy = _unpack(_pack(z.float()), N) * rstd, t["dy"].float()
        g = dy * t["gamma"].float()
        dx = t["dz"].float() + rstd * (g - xhat * (g * xhat).mean(dim=1, keepdim=True))
        return {"y": y.to(dtype), "rstd": rstd[:, 0], "dx": dx.to(dtype), "dgamma": (dy * xhat).sum(dim=0).to(t["gamma"].dtype)}
    if kind == "act_train":
        p = t["x"].float() + t["bias"].float()
        dx = t["dy"].float() * _act_gradient(_unpack(_pack(p), N), act)
        return {"y": _act(p, act).to(dtype), "dx": dx.to(dtype), "dbias": dx.sum(dim=0).to(t["bias"].dtype)}
    if kind == "keep":
        return {"y": _unpack(_pack(t["x"].float()), N).to(dtype)}
    if case["operands"] == "packed":
        a, b = _unpack(t["a"], K), _unpack(t["b"], K)
    else:
        a, b = t["a"].float(), t["b"].float()
    p = torch.mm(a, b.t())
    if case["bias"]:
        p = p + t["bias"].float()
    if kind == "product":
        out = _act(p, act)
        return {"out": (out + t["residual"].float() if case["residual"] else out).to(dtype)}
    dp = t["dh"].float() * _act_gradient(_unpack(_pack(p), N), act)
    dbias = dp.sum(dim=0).to(t["bias"].dtype)
    dp = dp.to(dtype)
    return {"out": _act(p, act).to(dtype), "dp": dp, "dbias": dbias, "dx": torch.mm(dp.float(), b).to(dtype),
            "dw": torch.mm(dp.float().t(), a).to(dtype)}


def _packed_bytes(rows, C):
    return rows * ((C + 31) // 32 * 32 + (C + 31) // 32)


def work(case):
    """Every input once and every output once, a checkpoint written and read; a norm takes some 6 operations an element and its
    gradient 10, a value into 8 bits or back 2, gelu some 20 and its gradient 30, silu 8 and 12."""
    kind, M, N, K = case["kind"], case["M"], case["N"], case["K"]
    size, params, n = _BYTES[case["dtype"]], _BYTES[case["params"]] * case["N"], M * N
    acts = {"none": (0, 0), "relu": (1, 1), "gelu": (20, 30), "silu": (8, 12)}[case["act"]]
    packed = _packed_bytes(M, N)
    if kind == "rms":
        return {"bytes": 4 * n * size + params, "flops": 6 * n}
    if kind == "rms_packed":
        return {"bytes": 3 * n * size + 2 * packed + 2 * n + params, "flops": 10 * n}
    if kind == "rms_train":
        return {"bytes": 6 * n * size + 2 * packed + 2 * params + 8 * M, "flops": 20 * n}
    if kind == "act_train":
        return {"bytes": 4 * n * size + 2 * packed + 2 * params, "flops": (6 + sum(acts)) * n}
    if kind == "keep":
        return {"bytes": 2 * n * size + 2 * packed, "flops": 4 * n}
    if kind == "feed":
        weights = _packed_bytes(K, N) + _packed_bytes(N, K)
        return {"bytes": 4 * n * size + 2 * packed + 2 * _packed_bytes(M, K) + weights + params, "flops": 4 * M * N * K + 8 * n + (acts[0] + 2) * M * K}
    operands = _packed_bytes(M, K) + _packed_bytes(N, K) if case["operands"] == "packed" else (M * K + N * K) * size
    vector = params if case["bias"] else 0
    if kind == "product":
        return {"bytes": operands + n * size * (2 if case["residual"] else 1) + vector, "flops": 2 * M * N * K + (acts[0] + 2) * n}
    # x and w are read by the forward pass, and again with what dp brings by the backward one
    return {"bytes": 3 * operands + 2 * packed + 2 * vector + 3 * n * size, "flops": 6 * M * N * K + (sum(acts) + 6) * n}


def _power(k):
    """2^k in 64 bits for whole k in 64 bits, from its pattern."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _e4m3(u):
    """64-bit values of at most 448 in size to the nearest multiple of their binade's eighth, ties to even."""
    binade = torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -20)))
    binade = binade + (u.abs() >= _power(binade + 1)).double() - (u.abs() < _power(binade)).double()
    step = _power(binade.clamp(min=-6.0) - 3)
    return torch.round(u / step) * step


def _kept(v):
    """What 64-bit values stand for once they are held in 8 bits, block by block."""
    out = torch.empty_like(v)
    C = v.shape[1]
    whole = C // 32 * 32
    for part, to in ((v[:, :whole].reshape(-1, 32), out[:, :whole]), (v[:, whole:], out[:, whole:])):
        if part.numel() == 0:
            continue
        most = part.abs().amax(dim=1, keepdim=True)
        k = torch.ceil(torch.log2((most / 448.0).clamp(min=2.0 ** -127))).clamp(min=-127.0)
        k = torch.where(448.0 * _power(k) < most, k + 1, k)
        k = torch.where((224.0 * _power(k) >= most) & (k > -127), k - 1, k)
        to.copy_((_e4m3(part / _power(k)) * _power(k)).reshape(to.shape))
    return out


def _meaning(packed, C):
    """What codes and scales stand for in 64 bits, from the bits themselves."""
    codes, scales = packed
    c = codes.long()
    sign, exponent, mantissa = 1 - 2 * (c >> 7), (c >> 3) & 15, (c & 7).double()
    value = sign * torch.where(exponent > 0, (8 + mantissa) * _power(exponent - 10), mantissa * 2.0 ** -9)
    return (value * _power(scales.long() - 127).repeat_interleave(32, dim=1)[:, :codes.shape[1]])[:, :C]


def _act_exact(v, act):
    """act and its derivative in 64 bits."""
    if act == "relu":
        return torch.where(v > 0, v, 0.0), (v > 0).double()
    if act == "gelu":
        upper = 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
        return v * upper, upper + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        upper = torch.sigmoid(v)
        return v * upper, upper + v * upper * torch.sigmoid(-v)
    return v, torch.ones_like(v)


def exact(case, seed):
    """The definitions in 64 bits."""
    t, kind, N, K, act = _inputs(case, seed), case["kind"], case["N"], case["K"], case["act"]
    dtype = _DTYPES[case["dtype"]]
    if kind == "keep":
        return {"y": _kept(t["x"].double())}
    if kind in ("rms", "rms_packed", "rms_train", "feed"):
        stored = (t["residual"].double() + t["x"].double()).float().to(dtype).double()  # z as it is stored
        root = ((stored ** 2).sum(dim=1) / N + case["eps"]).sqrt()
        gamma = t["gamma"].double()
        y = stored / root[:, None] * gamma
        z = t["residual"].double() + t["x"].double()
        if kind == "rms":
            return {"z": z, "y": y}
        if kind == "rms_packed":
            return {"z": z, "y": _kept(y)}
        if kind == "feed":
            h = _act_exact(_kept(y) @ _meaning(t["w1"], N).t(), act)[0]
            return {"z": z, "out": _kept(h) @ _meaning(t["w2"], K).t() + stored}
        z, dy = _kept(stored), t["dy"].double()
        along = (dy * gamma * z).sum(dim=1) / (N * root ** 3)
        return {"y": y, "rstd": 1 / root, "dx": t["dz"].double() + dy * gamma / root[:, None] - z * along[:, None],
                "dgamma": (dy * z / root[:, None]).sum(dim=0)}
    if kind == "act_train":
        p = (t["x"].double() + t["bias"].double()).float().double()  # the sum as it is kept
        dx = t["dy"].double() * _act_exact(_kept(p), act)[1]
        return {"y": _act_exact(p, act)[0], "dx": dx, "dbias": dx.sum(dim=0)}
    if case["operands"] == "packed":
        a, b = _meaning(t["a"], K), _meaning(t["b"], K)
    else:
        a, b = t["a"].double(), t["b"].double()
    p = a @ b.t()
    if case["bias"]:
        p = p + t["bias"].double()
    if kind == "product":
        out = _act_exact(p, act)[0]
        return {"out": out + t["residual"].double() if case["residual"] else out}
    dp = t["dh"].double() * _act_exact(_kept(p), act)[1]
    stored = dp.float().to(dtype).double()  # dp as it is stored, which the products read
    return {"out": _act_exact(p, act)[0], "dp": dp, "dbias": dp.sum(dim=0), "dx": stored @ b, "dw": stored.t() @ a}
