"""Activation checkpoints in 8 bits and the operators that write and read them, as cases that can be timed.

A case is one call, or one forward and backward pass, of a layer in data-parallel training on one GPU:

  op "checkpoint"  a matrix of activations encoded to 8 bits, and decoded again;
  op "pointwise"   an activation function (with or without a gate) that saves its inputs in 8 bits, and its backward pass;
  op "group_norm"  group norm with an activation, channels last, which may save its input in 8 bits;
  op "wgrad"       weight and bias gradient of a linear layer (or 1x1 convolution) from its 8-bit input.

Keys of a case: the sizes of the op, `dtype` of the activations ("f32", "f16", "bf16"), `act` ("none", "relu", "silu",
"gelu"), `dir` ("forward", "backward", "step": both), `gated`, `strided` (the inputs are column ranges of a wider matrix),
`saved` (the backward pass of the group norm reads the 8-bit input), `bias`.

The 8-bit form of a matrix [rows, cols]: groups of 32 columns of a row share one power of two 2^e, the smallest
with max|x| <= 127 * 2^e (-120 <= e <= 121); an element is the whole number nearest to x / 2^e.
"""
import math

import torch

own = False

GROUP = 32
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
MOST_ELEMS = 1 << 26   # elements of the largest listed matrix
MOST_MACS = 1 << 38    # products of the largest listed weight gradient


def _checkpoint(rows, cols, dtype):
    return {"op": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype}


def _pointwise(rows, cols, dtype, act, dir, gated=False, strided=False):
    return {"op": "pointwise", "rows": rows, "cols": cols, "dtype": dtype, "act": act, "dir": dir, "gated": gated, "strided": strided}


def _group_norm(N, P, C, G, dtype, act, dir, saved):
    return {"op": "group_norm", "N": N, "P": P, "C": C, "G": G, "dtype": dtype, "act": act, "dir": dir, "saved": saved}


def _wgrad(rows, cols, out_cols, dtype, bias):
    return {"op": "wgrad", "rows": rows, "cols": cols, "out_cols": out_cols, "dtype": dtype, "bias": bias}


def listed():
    cases = {
        # the input of a fully connected layer for one batch of 32 (latency and launches)
        "checkpoint_32x4096": _checkpoint(32, 4096, "bf16"),
        # a wide layer's input for 16,384 tokens
        "checkpoint_16384x4096": _checkpoint(16384, 4096, "bf16"),
        # rows that end inside a group and begin at any address
        "checkpoint_4099x1001": _checkpoint(4099, 1001, "f16"),
        # ReLU after a fully connected layer, fp32 training
        "relu_256x4096": _pointwise(256, 4096, "f32", "relu", "step"),
        # a gated unit whose two inputs are the halves of one product's rows
        "gated_silu_8192x8192": _pointwise(8192, 8192, "bf16", "silu", "step", gated=True, strided=True),
        # backward alone, a layer of no round width
        "gelu_backward_20011x1000": _pointwise(20011, 1000, "f16", "gelu", "backward"),
        # one image through the third stage of the 50-layer CNN, evaluation
        "norm_relu_1x196x1024": _group_norm(1, 196, 1024, 32, "bf16", "relu", "forward", False),
        # a batch of 32 at the end of its first stage, training with the input kept in 8 bits
        "norm_silu_32x3136x256": _group_norm(32, 3136, 256, 32, "bf16", "silu", "step", True),
        # few large images, fp32, the input kept as it is
        "norm_gelu_4x16384x256": _group_norm(4, 16384, 256, 32, "f32", "gelu", "step", False),
        # the classifier of the 19-layer CNN for a batch of 32
        "wgrad_32x4096x1000": _wgrad(32, 4096, 1000, "bf16", True),
        # a 1x1 convolution on 32 maps of 56 x 56: few weights, a long sum
        "wgrad_100352x64x256": _wgrad(100352, 64, 256, "bf16", False),
        # a wide square layer for 16,384 tokens
        "wgrad_16384x4096x4096": _wgrad(16384, 4096, 4096, "bf16", True),
    }
    return [{"name": name, **c} for name, c in cases.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _width(rng, lo, hi):
    """A width: round to 64, to 8, or anything."""
    w = _log(rng, lo, hi)
    r = rng.choice((64, 64, 8, 1))
    return max(lo, min(hi, (w + r - 1) // r * r))


def draw(rng):
    op = rng.choice(("checkpoint", "pointwise", "group_norm", "wgrad"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "checkpoint":
        cols = _width(rng, 1, 16384)
        return _checkpoint(_log(rng, 1, MOST_ELEMS // 2 // cols), cols, dtype)
    if op == "pointwise":
        cols = _width(rng, 1, 16384)
        rows = _log(rng, 1, MOST_ELEMS // 2 // cols)
        return _pointwise(rows, cols, dtype, rng.choice(("relu", "silu", "gelu")), rng.choice(("forward", "backward", "step")),
                          rng.random() < 0.5, rng.random() < 0.3)
    if op == "group_norm":
        per_group = rng.choice((1, 2, 3, 4, 5, 8, 10, 16, 32, 64))
        G = rng.choice((1, 8, 16, 32))
        C = G * per_group
        P = _log(rng, -(-64 // per_group), 16384)  # groups of 64 values and more: of two or three, the backward pass leaves rounding alone
        N = _log(rng, 1, max(1, min(64, MOST_ELEMS // 2 // (P * C))))
        dir = rng.choice(("forward", "backward", "step"))
        # the derivative of ReLU jumps where the normalised value is 0, so it is drawn for the forward pass alone: no two ways
        # to round a sum put all of 10^7 values on the same side
        act = rng.choice(("none", "relu", "silu", "gelu") if dir == "forward" else ("none", "silu", "gelu"))
        return _group_norm(N, P, C, G, dtype, act, dir, rng.random() < 0.6)
    cols, out_cols = _width(rng, 8, 4096), _width(rng, 8, 4096)
    rows = _log(rng, 1, min(100352, MOST_MACS // 4 // (cols * out_cols)))
    return _wgrad(rows, cols, out_cols, dtype, rng.random() < 0.5)


def _groups(cols):
    return -(-cols // GROUP)


def work(case):
    b = BYTES[case["dtype"]]
    op = case["op"]
    if op == "group_norm":
        E, saved = case["N"] * case["P"] * case["C"], case["N"] * case["P"] * (case["C"] + _groups(case["C"]))
        bytes_ = 0
        if case["dir"] in ("forward", "step"):
            bytes_ += 2 * E * b + (saved if case["saved"] else 0)
        if case["dir"] in ("backward", "step"):
            bytes_ += 2 * E * b + (saved if case["saved"] else E * b)
        return {"bytes": bytes_ + 16 * case["C"], "flops": 20 * E}
    rows, cols = case["rows"], case["cols"]
    E, saved = rows * cols, rows * (cols + _groups(cols))
    if op == "checkpoint":
        return {"bytes": 2 * (E * b + saved), "flops": 4 * E}
    if op == "pointwise":
        n = 2 if case["gated"] else 1
        bytes_ = 0
        if case["dir"] in ("forward", "step"):
            bytes_ += n * E * b + E * b + n * saved
        if case["dir"] in ("backward", "step"):
            bytes_ += E * b + n * saved + n * E * b
        return {"bytes": bytes_, "flops": 20 * n * E}
    out = case["out_cols"]
    return {"bytes": rows * out * b + saved + 4 * cols * out, "flops": 2 * rows * cols * out}


# ----------------------------------------------------------------------------------------------------------------
# inputs

def _values(gen, shape, dtype, scale=1.0):
    """Activations: normal, with a scale of its own per channel, so that groups hold small values beside large ones."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x *= torch.exp(0.7 * torch.randn(shape[-1], device="cuda", generator=gen)) * scale
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    op = case["op"]
    st = dict(case)
    new = lambda *shape, dtype=dt: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
    if op == "group_norm":
        N, P, C, G = case["N"], case["P"], case["C"], case["G"]
        x = (_values(gen, (N, P, C), torch.float32) + 1 + 0.5 * torch.randn(C, device="cuda", generator=gen)).to(dt)
        st["gamma"] = 1 + 0.2 * torch.randn(C, device="cuda", generator=gen)
        st["beta"] = 0.2 * torch.randn(C, device="cuda", generator=gen)
        st["eps"] = 1e-5
        st["mean"], st["rstd"] = new(N, G, dtype=torch.float32), new(N, G, dtype=torch.float32)
        st["codes"], st["scales"] = new(N * P, C, dtype=torch.int8), new(N * P, _groups(C), dtype=torch.uint8)
        if case["dir"] != "forward":
            st["dy"] = _values(gen, (N, P, C), dt, 0.1)
            st["dx"], st["dgamma"], st["dbeta"] = new(N, P, C), new(C, dtype=torch.float32), new(C, dtype=torch.float32)
        if case["dir"] != "backward":
            st["y"] = new(N, P, C)
        else:  # what an earlier forward pass left
            st["mean"], st["rstd"] = _group_stats(x, G, st["eps"])
            if case["saved"]:
                st["codes"], st["scales"] = _encode(x.view(N * P, C))
        if case["dir"] != "backward" or not case["saved"]:
            st["x"] = x
        st["ws"] = new(_ws_group_norm(N, P, C), dtype=torch.uint8)
        return st
    rows, cols = case["rows"], case["cols"]
    if op == "checkpoint":
        st["x"], st["y"] = _values(gen, (rows, cols), dt), new(rows, cols)
        st["codes"], st["scales"] = new(rows, cols, dtype=torch.int8), new(rows, _groups(cols), dtype=torch.uint8)
        return st
    if op == "pointwise":
        n = 2 if case["gated"] else 1
        ld = 2 * cols if case["strided"] else cols
        names = ("x", "up")[:n]
        wide = [_values(gen, (rows, ld), dt) for _ in range(1 if case["strided"] else n)]
        dwide = [torch.zeros(rows, ld, device="cuda", dtype=dt) for _ in wide]
        for k, name in enumerate(names):
            if case["strided"]:
                st[name], st["d" + name] = wide[0][:, k * cols:(k + 1) * cols], dwide[0][:, k * cols:(k + 1) * cols]
            else:
                st[name], st["d" + name] = wide[k], dwide[k]
            if case["dir"] == "backward":
                st[name + "_codes"], st[name + "_scales"] = _encode(st[name])
            else:
                st[name + "_codes"], st[name + "_scales"] = new(rows, cols, dtype=torch.int8), new(rows, _groups(cols), dtype=torch.uint8)
        st["y"] = new(rows, cols)
        st["dy"] = _values(gen, (rows, cols), dt, 0.1)
        st["ld"] = ld
        if case["dir"] == "backward":
            for name in names:
                del st[name]
        return st
    out = case["out_cols"]
    st["codes"], st["scales"] = _encode(_values(gen, (rows, cols), dt))
    st["dy"] = _values(gen, (rows, out), dt, 0.1)
    st["dw"], st["db"] = new(out, cols, dtype=torch.float32), new(out, dtype=torch.float32)
    st["ws"] = new(WS_WGRAD, dtype=torch.uint8)
    return st


# scratch that the framework's calls are given, enough for any case here (a training loop keeps one such buffer)
WS_WGRAD = 96 << 20


def _ws_group_norm(N, P, C):
    return (1 << 20) + 64 * N * C * (1 + P // 64)


# ----------------------------------------------------------------------------------------------------------------
# plain forms

def _encode(x):
    rows, cols = x.shape
    g = _groups(cols)
    v = torch.nn.functional.pad(x.float(), (0, g * GROUP - cols)).view(rows, g, GROUP)
    amax = v.abs().amax(2)
    fine = torch.isfinite(amax)
    m, ex = torch.frexp(torch.where(fine & (amax > 0), amax, torch.ones_like(amax)))
    e = (ex - 7 + (m > 127 / 128)).clamp(-120, 121)
    e = torch.where(amax > 0, e, torch.full_like(e, -120))
    inv = ((127 - e) << 23).view(torch.float32)
    q = torch.round(v * inv[:, :, None]).clamp(-127, 127)
    q = torch.where(fine[:, :, None], q, torch.zeros_like(q))
    scales = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return q.view(rows, g * GROUP)[:, :cols].to(torch.int8).contiguous(), scales


def _decode(codes, scales):
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * s.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _group_stats(x, G, eps):
    N, P, C = x.shape
    v = x.float().view(N, P, G, C // G)
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, 1 / torch.sqrt(var + eps)


def _plain_group_norm(st):
    N, P, C, G, act, dt = st["N"], st["P"], st["C"], st["G"], st["act"], DTYPES[st["dtype"]]
    got = {}
    wide = lambda s: s.repeat_interleave(C // G, 1)[:, None, :]  # noqa: E731
    mean, rstd, codes, scales = st["mean"], st["rstd"], st["codes"], st["scales"]
    if st["dir"] != "backward":
        mean, rstd = _group_stats(st["x"], G, st["eps"])
        z = (st["x"].float() - wide(mean)) * wide(rstd) * st["gamma"] + st["beta"]
        got["y"] = _act(z, act).to(dt)
        got["mean"], got["rstd"] = mean, rstd
        if st["saved"]:
            codes, scales = _encode(st["x"].view(N * P, C))
    if st["dir"] != "forward":
        xv = _decode(codes, scales).view(N, P, C) if st["saved"] else st["x"].float()
        xh = (xv - wide(mean)) * wide(rstd)
        dz = st["dy"].float() * _act_slope(xh * st["gamma"] + st["beta"], act)
        got["dgamma"], got["dbeta"] = (dz * xh).sum((0, 1)), dz.sum((0, 1))
        gz = dz * st["gamma"]
        m1 = gz.view(N, P, G, C // G).mean((1, 3))
        m2 = (gz * xh).view(N, P, G, C // G).mean((1, 3))
        got["dx"] = (wide(rstd) * (gz - wide(m1) - xh * wide(m2))).to(dt)
    elif st["saved"]:
        got["kept"] = _decode(codes, scales).to(torch.bfloat16)
    return got


def _plain_pointwise(st):
    act, dt, gated = st["act"], DTYPES[st["dtype"]], st["gated"]
    got = {}
    kept = {n: (st[n + "_codes"], st[n + "_scales"]) for n in (("x", "up") if gated else ("x",))}
    if st["dir"] != "backward":
        y = _act(st["x"].float(), act)
        got["y"] = (y * st["up"].float() if gated else y).to(dt)
        kept = {n: _encode(st[n]) for n in kept}
    if st["dir"] != "forward":
        x, dy = _decode(*kept["x"]), st["dy"].float()
        if gated:
            got["dup"] = (dy * _act(x, act)).to(dt)
            dy = dy * _decode(*kept["up"])
        got["dx"] = (dy * _act_slope(x, act)).to(dt)
    else:
        got.update({"kept_" + n: _decode(*k).to(torch.bfloat16) for n, k in kept.items()})
    return got


def _plain(st):
    if st["op"] == "checkpoint":
        return {"y": _decode(*_encode(st["x"])).to(DTYPES[st["dtype"]])}
    if st["op"] == "pointwise":
        return _plain_pointwise(st)
    if st["op"] == "group_norm":
        return _plain_group_norm(st)
    dy = st["dy"].float()
    got = {"dw": dy.t() @ _decode(st["codes"], st["scales"])}
    if st["bias"]:
        got["db"] = dy.sum(0)
    return got


# ----------------------------------------------------------------------------------------------------------------
# the framework's calls

def _own(st):
    import paper_2002_11082_b200 as ogq

    dt = {"f32": ogq.OGQ_F32, "f16": ogq.OGQ_F16, "bf16": ogq.OGQ_BF16}[st["dtype"]]
    op = st["op"]
    nearest = ogq.OGQ_ROUND_NEAREST
    if op == "checkpoint":
        rows, cols = st["rows"], st["cols"]
        ogq.ogq_act8_encode(st["x"], cols, rows, cols, dt, nearest, 0, 0, st["codes"], st["scales"])
        ogq.ogq_act8_decode(st["codes"], st["scales"], rows, cols, dt, st["y"], cols)
        return {"y": st["y"]}
    if op == "wgrad":
        db = st["db"] if st["bias"] else None
        ogq.ogq_act8_wgrad(st["dy"], st["out_cols"], st["codes"], st["scales"], st["rows"], st["cols"], st["out_cols"], dt, 0,
                           st["dw"], db, st["ws"], st["ws"].numel())
        return {"dw": st["dw"], "db": db} if st["bias"] else {"dw": st["dw"]}
    act = {"none": ogq.OGQ_ACT_NONE, "relu": ogq.OGQ_ACT_RELU, "silu": ogq.OGQ_ACT_SILU, "gelu": ogq.OGQ_ACT_GELU}[st["act"]]
    got = {}
    if op == "pointwise":
        rows, cols, ld, gated = st["rows"], st["cols"], st["ld"], st["gated"]
        up_codes, up_scales = (st["up_codes"], st["up_scales"]) if gated else (None, None)
        if st["dir"] != "backward":
            ogq.ogq_act8_forward(st["x"], ld, st["up"] if gated else None, ld, rows, cols, dt, act, nearest, 0, 0, st["y"], cols,
                                 st["x_codes"], st["x_scales"], up_codes, up_scales)
            got["y"] = st["y"]
        if st["dir"] != "forward":
            ogq.ogq_act8_backward(st["dy"], cols, st["x_codes"], st["x_scales"], up_codes, up_scales, rows, cols, dt, act,
                                  st["dx"], ld, st["dup"] if gated else None, ld)
            got.update({"dx": st["dx"], "dup": st["dup"]} if gated else {"dx": st["dx"]})
        else:
            for n in (("x", "up") if gated else ("x",)):
                kept = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
                ogq.ogq_act8_decode(st[n + "_codes"], st[n + "_scales"], rows, cols, ogq.OGQ_BF16, kept, cols)
                got["kept_" + n] = kept
        return got
    N, P, C, G = st["N"], st["P"], st["C"], st["G"]
    codes, scales = (st["codes"], st["scales"]) if st["saved"] else (None, None)
    if st["dir"] != "backward":
        ogq.ogq_group_norm_forward(st["x"], N, P, C, G, dt, st["gamma"], st["beta"], st["eps"], act, nearest, 0, 0, st["y"],
                                   st["mean"], st["rstd"], codes, scales, st["ws"], st["ws"].numel())
        got.update({"y": st["y"], "mean": st["mean"], "rstd": st["rstd"]})
    if st["dir"] != "forward":
        ogq.ogq_group_norm_backward(st["dy"], None if st["saved"] else st["x"], codes, scales, N, P, C, G, dt, st["gamma"], st["beta"],
                                    act, st["mean"], st["rstd"], st["dx"], st["dgamma"], st["dbeta"], st["ws"], st["ws"].numel())
        got.update({"dx": st["dx"], "dgamma": st["dgamma"], "dbeta": st["dbeta"]})
    elif st["saved"]:
        kept = torch.empty(N * P, C, device="cuda", dtype=torch.bfloat16)
        ogq.ogq_act8_decode(codes, scales, N * P, C, ogq.OGQ_BF16, kept, C)
        got["kept"] = kept
    return got


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _kept64(x):
    """x of shape [rows, cols] as its 8-bit form gives it back."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    whole = cols // GROUP * GROUP
    for lo, hi in ((0, whole), (whole, cols)):
        if hi > lo:
            v = x[:, lo:hi].double().reshape(rows, -1, GROUP if lo == 0 and whole else hi - lo)
            top = v.abs().max(2, keepdim=True).values
            e = torch.floor(torch.log2(top / 127)).clamp(-122, 121) - 1
            for _ in range(3):  # up to the first power of two that is not below top / 127
                e += 127 * torch.ldexp(torch.ones_like(e), e.int()) < top
            e = e.clamp(-120, 121)
            unit = torch.ldexp(torch.ones_like(e), e.int())
            out[:, lo:hi] = (torch.round(v / unit).clamp(-127, 127) * unit).reshape(rows, hi - lo)
    return out


def _given64(codes, scales):
    unit = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.int() - 127)
    at = torch.arange(codes.shape[1], device=codes.device) // GROUP
    return codes.double() * unit[:, at]


def _f64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z * 1


def _slope64(z, act):
    z = z.detach().requires_grad_()
    return torch.autograd.grad(_f64(z, act).sum(), z)[0]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    got = {}
    if op == "checkpoint":
        return {"y": _kept64(st["x"])}
    if op == "wgrad":
        dy = st["dy"].double()
        got["dw"] = torch.einsum("to,ti->oi", dy, _given64(st["codes"], st["scales"]))
        if case["bias"]:
            got["db"] = dy.sum(0)
        return got
    act = case["act"]
    if op == "pointwise":
        names = ("x", "up") if case["gated"] else ("x",)
        if case["dir"] != "backward":
            y = _f64(st["x"].double(), act)
            got["y"] = y * st["up"].double() if case["gated"] else y
            del y
            kept = {n: _kept64(st[n]) for n in names}
        else:
            kept = {n: _given64(st[n + "_codes"], st[n + "_scales"]) for n in names}
        if case["dir"] != "forward":
            dy = st["dy"].double()
            got["dx"] = dy * _slope64(kept["x"], act)
            if case["gated"]:
                got["dx"] *= kept["up"]
                got["dup"] = dy * _f64(kept["x"], act)
        else:
            got.update({"kept_" + n: k for n, k in kept.items()})
        return got
    N, P, C, G = (case[k] for k in "NPCG")
    per = C // G
    gamma, beta = st["gamma"].double(), st["beta"].double()
    mean, rstd = st["mean"].double(), st["rstd"].double()
    kept = None
    if case["dir"] != "backward":
        x = st["x"].double().transpose(1, 2).reshape(N, G, per * P)
        mean = x.sum(2) / (per * P)
        rstd = (((x - mean[:, :, None]) ** 2).sum(2) / (per * P) + st["eps"]) ** -0.5
        xh = ((x - mean[:, :, None]) * rstd[:, :, None]).reshape(N, C, P)
        got["y"] = _f64(gamma[:, None] * xh + beta[:, None], act).transpose(1, 2)
        got["mean"], got["rstd"] = mean, rstd
        del x, xh
        if case["saved"]:
            kept = _kept64(st["x"].reshape(N * P, C)).reshape(N, P, C)
    elif case["saved"]:
        kept = _given64(st["codes"], st["scales"]).reshape(N, P, C)
    if case["dir"] == "forward":
        if case["saved"]:
            got["kept"] = kept.reshape(N * P, C)
        return got
    x = (kept if case["saved"] else st["x"].double()).transpose(1, 2).reshape(N, G, per, P)
    xh = (x - mean[:, :, None, None]) * rstd[:, :, None, None]
    gamma, beta = gamma.reshape(G, per, 1), beta.reshape(G, per, 1)
    dz = st["dy"].double().transpose(1, 2).reshape(N, G, per, P) * _slope64(gamma * xh + beta, act)
    got["dgamma"] = (dz * xh).sum((0, 3)).reshape(C)
    got["dbeta"] = dz.sum((0, 3)).reshape(C)
    t = gamma * dz
    dx = t - t.mean((2, 3), keepdim=True) - xh * (t * xh).mean((2, 3), keepdim=True)
    got["dx"] = (dx * rstd[:, :, None, None]).reshape(N, C, P).transpose(1, 2)
    return got
