"""Group norm with an activation on channels-last images, and microscaled 4-bit products: what they are timed with.

The sizes are those of the residual networks in bottleneck.py (56x56 down to 7x7, 64 to 2048 channels), of the large-image
set, and of a generic square product; ``draw`` spreads over the same ranges.  Kinds of case:

* ``norm``: y = act(group_norm(x) gamma + beta + residual), x [batch][H][W][C], perhaps a slice of wider pixels (``pitch``);
* ``norm_backward``: its gradients of x, gamma, beta and the residual, from the statistics that the forward pass saved;
* ``round_trip``: x to 4 bits (blocks of 32 channels, e2m1 values, a power of two each) and back;
* ``conv``: a 1x1 convolution with weights in 4 bits, which takes x in floating point and quantises it itself;
* ``norm_conv``: the norm that writes 4 bits, and the 1x1 convolution that reads them;
* ``product``: rows times rows, both already in 4 bits.

``call`` says how the user's program calls: ``bound`` through the zero-argument launcher on fixed buffers (a serving loop),
``fresh`` with new output tensors every time.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _norm_case(kind, batch, H, W, C, groups, act, dtype, residual=False, pitch=0, call="fresh"):
    return {"kind": kind, "batch": batch, "H": H, "W": W, "C": C, "groups": groups, "act": act, "dtype": dtype,
            "residual": residual, "pitch": pitch or C, "call": call}


def _conv_case(kind, batch, H, W, C, N, stride, act, dtype, residual=False, call="fresh", groups=0):
    return {"kind": kind, "batch": batch, "H": H, "W": W, "C": C, "N": N, "stride": stride, "act": act, "dtype": dtype,
            "residual": residual, "call": call, "groups": groups}


def listed():
    cases = {
        # One image at the end of a residual network in a serving loop: the smallest call, all launch and latency.
        "norm_b1_7": _norm_case("norm", 1, 7, 7, 512, 32, "relu", "fp32", call="bound"),
        # Nothing divides anything: odd image, 15 channels to a group, a slice of the wider pixels of a concatenation.
        "norm_b3_ragged": _norm_case("norm", 3, 37, 29, 150, 10, "silu", "bf16", pitch=250),
        # The end of a bottleneck block of a batch, with its shortcut: the largest norm.
        "norm_b32_56": _norm_case("norm", 32, 56, 56, 256, 32, "relu", "fp32", residual=True),
        # One large image, as at the outer levels of a network that makes images: few groups, much of each.
        "norm_b1_224": _norm_case("norm", 1, 224, 224, 64, 32, "silu", "fp16"),
        # Training: a batch's share at 28x28 with its shortcut, and the wide 56x56 stage in 16 bits.
        "backward_b8_28": _norm_case("norm_backward", 8, 28, 28, 512, 32, "silu", "fp32", residual=True),
        "backward_b32_56": _norm_case("norm_backward", 32, 56, 56, 256, 32, "silu", "bf16"),
        # Activations put away in 4 bits and read back: ragged pixels in 16 bits, and a whole stage in fp32.
        "round_trip_ragged": {"kind": "round_trip", "rows": 3219, "cols": 150, "dtype": "bf16"},
        "round_trip_b32_56": {"kind": "round_trip", "rows": 100352, "cols": 256, "dtype": "fp32"},
        # The classifier of one image: a single row against the weights.
        "conv_one_row": _conv_case("conv", 1, 1, 1, 2048, 1000, 1, "none", "fp32", call="bound"),
        # The projection shortcut of a stage's first block, every second pixel each way.
        "conv_b32_56_s2": _conv_case("conv", 32, 56, 56, 256, 512, 2, "none", "fp32"),
        # The last third of a bottleneck block normalised by groups: norm + activation, 1x1 to four times the width, shortcut.
        "norm_conv_b32_28": _conv_case("norm_conv", 32, 28, 28, 128, 512, 1, "relu", "bf16", residual=True, groups=32),
        # A square product that the matrix cores bound.
        "product_8192": {"kind": "product", "M": 8192, "N": 8192, "K": 8192, "dtype": "bf16"},
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm_backward", "round_trip", "conv", "conv", "norm_conv", "product"))
    dtype = rng.choice(tuple(DTYPES))
    while True:
        if kind == "product":
            case = {"kind": kind, "M": _log_int(rng, 1, 8192), "N": _log_int(rng, 10, 8192), "K": _log_int(rng, 20, 8192), "dtype": dtype}
        elif kind == "round_trip":
            case = {"kind": kind, "rows": _log_int(rng, 1, 200000), "cols": _log_int(rng, 4, 2048), "dtype": dtype}
        else:
            batch, H = _log_int(rng, 1, 64), _log_int(rng, 1 if kind == "conv" else 7, 224)
            W = H if rng.random() < 0.7 else max(1, min(224, int(H * rng.uniform(0.6, 1.6))))
            groups = rng.choice((1, 4, 8, 16, 32, 32, 32, 64))
            C = groups * _log_int(rng, 1, 64)
            if kind == "conv":
                C = _log_int(rng, 20, 2048)
            act, call = rng.choice(("none", "relu", "silu")), rng.choice(("bound", "fresh"))
            if kind == "norm_backward" and act == "relu":
                act = "silu"     # the border of a ReLU falls differently for every order of summation
            if kind in ("norm", "norm_backward"):
                pitch = C + rng.choice((0, 0, 0, 8, _log_int(rng, 1, 256)))
                case = _norm_case(kind, batch, H, W, C, groups, act, dtype, rng.random() < 0.4, pitch, "fresh" if kind == "norm_backward" else call)
            else:
                # Behind a norm a value next to the border of two 4-bit values may fall to either: outputs in 16 bits.
                dt = dtype if kind == "conv" else rng.choice(("bf16", "fp16"))
                case = _conv_case(kind, batch, H, W, C, _log_int(rng, 10, 2048), rng.choice((1, 1, 2)) if kind == "conv" else 1, act, dt,
                                  rng.random() < 0.4, call, groups if kind == "norm_conv" else 0)
            if C < 4 or C > 2048:
                continue
        w = work(case)
        if w["bytes"] <= 250e6 and w["flops"] <= 1e12:
            return case


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def _out(case):
    return -(-case["H"] // case["stride"]), -(-case["W"] // case["stride"])


def _mx4_bytes(rows, cols):
    return rows * -(-cols // 32) * 17


def work(case):
    kind, e = case["kind"], _size(case["dtype"])
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": _mx4_bytes(M, K) + _mx4_bytes(N, K) + 4 * N + e * M * N, "flops": 2 * M * N * K}
    if kind == "round_trip":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * (e * n + _mx4_bytes(case["rows"], case["cols"])), "flops": 4 * n}
    pixels = case["batch"] * case["H"] * case["W"]
    n = pixels * case["C"]
    if kind == "norm":
        return {"bytes": e * n * (3 if case["residual"] else 2) + 8 * case["C"], "flops": 10 * n}
    if kind == "norm_backward":
        return {"bytes": e * n * (5 if case["residual"] else 3) + 16 * case["C"] + 8 * case["batch"] * case["groups"], "flops": 25 * n}
    Ho, Wo = _out(case)
    rows, N = case["batch"] * Ho * Wo, case["N"]
    read = pixels if kind == "norm_conv" else rows
    more = 8 * case["C"] if kind == "norm_conv" else 0
    return {"bytes": e * read * case["C"] + _mx4_bytes(N, case["C"]) + 4 * N + more + e * rows * N * (2 if case["residual"] else 1),
            "flops": 2 * rows * N * case["C"] + (10 * n if kind == "norm_conv" else 0)}


def _pixels(case, normal, pitch):
    """Activations as they leave a convolution, every channel with a level and a spread of its own."""
    C = case["C"]
    wide = normal((case["batch"], case["H"], case["W"], pitch))
    wide = wide * (0.5 + torch.rand_like(wide[0, 0, 0])) + 0.5 * torch.randn_like(wide[0, 0, 0])
    return wide.to(DTYPES[case["dtype"]])[..., :C]


def prepare(case, seed):
    device = torch.device("cuda", 0)
    gen = torch.Generator(device=device).manual_seed(int(seed))
    torch.cuda.manual_seed(int(seed))

    def normal(shape, scale=1.0):
        return torch.randn(shape, device=device, generator=gen) * scale

    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    state = {"case": case, "dtype": dtype}
    if kind == "round_trip":
        state["x"] = (normal((case["rows"], case["cols"])) * (0.5 + 2 * torch.rand((case["rows"], 1), device=device, generator=gen))).to(dtype)
        return state
    if kind == "product":
        for key, rows in (("a", case["M"]), ("b", case["N"])):
            blocks = -(-case["K"] // 32)
            codes = torch.randint(0, 256, (rows, blocks * 16), device=device, generator=gen, dtype=torch.uint8)
            ragged = case["K"] - 32 * (blocks - 1)             # what lies behind the last value is zero
            last = torch.arange(16, device=device)
            codes[:, -16:] &= (0x0f * (2 * last < ragged) + 0xf0 * (2 * last + 1 < ragged)).to(torch.uint8)
            scales = torch.randint(118, 124, (rows, blocks), device=device, generator=gen, dtype=torch.uint8)
            state[key] = (codes, scales)
        state["bias"] = normal((case["N"],), 0.1)
        return state
    C = case["C"]
    state["x"] = _pixels(case, normal, case.get("pitch", C))
    image = (case["batch"], case["H"], case["W"])
    if kind != "conv":
        state["gamma"], state["beta"] = 1 + 0.2 * normal((C,)), 0.2 * normal((C,))
    if kind in ("norm", "norm_backward"):
        state["residual"] = normal(image + (C,)).to(dtype) if case["residual"] else None
    if kind == "norm_backward":
        state["dy"] = normal(image + (C,)).to(dtype)
        state["stats"] = _statistics(state["x"], case["groups"])
    if kind in ("conv", "norm_conv"):
        Ho, Wo = _out(case)
        state["weights"] = normal((C, case["N"], 1, 1), C ** -0.5)
        state["values"] = _plain_mx4(state["weights"].reshape(C, case["N"]).t())    # kept in 4 bits' values: [N][C]
        state["bias"] = normal((case["N"],), 0.1)
        state["residual"] = normal((case["batch"], Ho, Wo, case["N"])).to(dtype) if case["residual"] else None
    if own:
        _prepare_own(state)
    return state


def _prepare_own(state):
    """The objects that a user's program keeps: plans with their workspaces and packed weights, launchers on fixed buffers."""
    case, x = state["case"], state["x"]
    if case["kind"] != "conv":
        from paper_2211_03715_amd.norm import GroupNorm
        act = "relu" if case["kind"] == "norm_conv" else case["act"]
        state["norm"] = GroupNorm(case["batch"], case["H"], case["W"], case["C"], case["groups"], eps=EPS, act=act, dtype=state["dtype"])
    if case["kind"] in ("conv", "norm_conv"):
        from paper_2211_03715_amd.mx4 import MX4Conv2d
        from paper_2211_03715_amd.workloads import Layer
        layer = Layer(case["batch"], case["C"], case["N"], case["H"], case["W"], 1, 1, 1, case["stride"], 0)
        state["conv"] = MX4Conv2d(layer, dtype=state["dtype"])
        state["conv"].pack(state["weights"])
    if case["call"] == "bound":
        if case["kind"] == "norm":
            state["y"] = torch.empty(x.shape, device=x.device, dtype=state["dtype"])
            state["launch"] = state["norm"].bind(x, state["y"], state["gamma"], state["beta"], residual=state["residual"])
        else:
            state["y"] = torch.empty(state["conv"].out_shape(), device=x.device, dtype=state["dtype"])
            extra = {"bias": state["bias"], "residual": state["residual"], "act": case["act"]}
            if case["kind"] == "conv":
                state["launch"] = state["conv"].bind(x, state["y"], **extra)
            else:
                q = state["norm"].new_quantized()
                first = state["norm"].bind_quantized(x, q, state["gamma"], state["beta"])
                second = state["conv"].bind(q, state["y"], **extra)
                state["launch"] = lambda: (first(), second())


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, kind = state["case"], state["case"]["kind"]
    if "launch" in state:
        state["launch"]()
        return state["y"]
    if kind == "norm":
        return state["norm"](state["x"], state["gamma"], state["beta"], residual=state["residual"])
    if kind == "norm_backward":
        dx, dgamma, dbeta, dres = state["norm"].backward(state["x"], state["dy"], state["stats"], state["gamma"], state["beta"], residual=state["residual"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta, "dresidual": dres}
    if kind in ("conv", "norm_conv"):
        x = state["x"] if kind == "conv" else state["norm"].quantized(state["x"], state["gamma"], state["beta"])
        return state["conv"](x, bias=state["bias"], residual=state["residual"], act=case["act"])
    from paper_2211_03715_amd import mx4
    if kind == "round_trip":
        return mx4.dequantize(*mx4.quantize(state["x"]), case["cols"], dtype=state["dtype"])
    return mx4.matmul(state["a"], state["b"], case["K"], bias=state["bias"], dtype=state["dtype"])


# ---- the plain form: elementary operations in fp32, rounded once

def _statistics(x, groups):
    B, C = x.shape[0], x.shape[-1]
    v = x.float().reshape(B, -1, groups, C // groups)
    mean = v.mean((1, 3), keepdim=True)
    var = (v - mean).square().mean((1, 3))
    return mean.reshape(B, groups), torch.rsqrt(var + EPS)


def _normalised(x, stats):
    mean, rstd = stats
    B, C = x.shape[0], x.shape[-1]
    v = x.float().reshape(B, -1, mean.shape[1], C // mean.shape[1])
    return ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)


def _activate(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    return v / (1 + torch.exp(-v)) if act == "silu" else v


def _plain_mx4(x):
    """The values that x has in 4 bits, in fp32: blocks of 32 along the last dimension."""
    C = x.shape[-1]
    v = torch.nn.functional.pad(x.float(), (0, -C % 32)).reshape(*x.shape[:-1], -1, 32)
    amax = v.abs().amax(-1, keepdim=True)
    shared = torch.clamp(torch.frexp(amax).exponent - 3, -127, 127)        # frexp: amax = m 2^e, m in [1/2, 1)
    shared = torch.where(amax > 0, shared, torch.full_like(shared, -127))
    up = ((127 - shared) << 23).view(torch.float32)                        # 2^-shared
    down = torch.where(shared > -127, ((shared + 127) << 23).view(torch.float32), torch.full_like(amax, 2.0 ** -127))
    a = v.abs() * up
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    q = torch.tensor(E2M1, device=x.device)[code]
    return (torch.where(v < 0, -q, q) * down).reshape(*x.shape[:-1], -1)[..., :C]


def _plain_values(codes, scales, cols):
    """The values of codes (two to a byte, the low half first) and scales, in fp32."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    nibbles = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1, 32).int()
    return (table[nibbles] * (scales.int() << 23).view(torch.float32)[..., None]).reshape(codes.shape[0], -1)[:, :cols]


def _run_plain(state):
    case, kind, dtype = state["case"], state["case"]["kind"], state["dtype"]
    if kind == "round_trip":
        return _plain_mx4(state["x"]).to(dtype)
    if kind == "product":
        a, b = (_plain_values(*state[k], case["K"]) for k in ("a", "b"))
        return (torch.matmul(a, b.t()) + state["bias"]).to(dtype)
    x = state["x"]
    if kind == "norm_backward":
        return _plain_backward(state)
    if kind != "conv":
        pre = _normalised(x, _statistics(x, case["groups"])) * state["gamma"] + state["beta"]
    if kind == "norm":
        pre = pre if state["residual"] is None else pre + state["residual"].float()
        return _activate(pre, case["act"]).to(dtype)
    v = _activate(pre, "relu") if kind == "norm_conv" else x[:, ::case["stride"], ::case["stride"]].float()
    y = torch.matmul(_plain_mx4(v), state["values"].t()) + state["bias"]
    y = y if state["residual"] is None else y + state["residual"].float()
    return _activate(y, case["act"]).to(dtype)


def _plain_backward(state):
    case, x, dtype = state["case"], state["x"], state["dtype"]
    xhat = _normalised(x, state["stats"])
    d = state["dy"].float()
    if case["act"] == "silu":
        pre = xhat * state["gamma"] + state["beta"]
        pre = pre if state["residual"] is None else pre + state["residual"].float()
        s = 1 / (1 + torch.exp(-pre))
        d = d * (s * (1 + pre * (1 - s)))
    B, C, G = x.shape[0], x.shape[-1], case["groups"]
    g, h = ((v * state["gamma"]).reshape(B, -1, G, C // G) for v in (d, d * xhat))
    m1, m2 = g.mean((1, 3), keepdim=True), h.mean((1, 3), keepdim=True)
    dx = state["stats"][1][:, None, :, None] * (g - m1 - xhat.reshape(g.shape) * m2)
    return {"dx": dx.reshape(x.shape).to(dtype), "dgamma": (d * xhat).sum((0, 1, 2)), "dbeta": d.sum((0, 1, 2)),
            "dresidual": d.to(dtype) if case["residual"] else None}


# ---- the definition in 64 bits

def _exact_act(v, act):
    return v.clamp(min=0) if act == "relu" else v * torch.sigmoid(v) if act == "silu" else v


def _exact_norm(x, gamma, beta, groups):
    B, H, W, C = x.shape
    v = x.double().permute(0, 3, 1, 2).reshape(B, groups, -1)
    var, mean = torch.var_mean(v, dim=2, unbiased=False, keepdim=True)
    v = ((v - mean) / torch.sqrt(var + EPS)).reshape(B, C, H, W).permute(0, 2, 3, 1)
    return v * gamma.double() + beta.double()


def _exact_mx4(x):
    C = x.shape[-1]
    v = torch.cat((x.double(), x.new_zeros(*x.shape[:-1], -C % 32, dtype=torch.float64)), -1).reshape(-1, 32)
    top = v.abs().amax(1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    e = torch.where(torch.pow(2.0, e) > top, e - 1, torch.where(torch.pow(2.0, e + 1) <= top, e + 1, e))
    scale = torch.pow(2.0, torch.where(top > 0, e - 2, torch.full_like(e, -127)).clamp(-127, 127))
    a = (v.abs() / scale).clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(a.dtype)
    return (torch.sign(v) * step * torch.round(a / step) * scale).reshape(*x.shape[:-1], -1)[..., :C]


def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "round_trip":
        return _exact_mx4(state["x"])
    if kind == "product":
        values = []
        for codes, scales in (state["a"], state["b"]):
            n = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.int64, device=codes.device)
            n[:, 0::2], n[:, 1::2] = codes % 16, codes // 16
            m, e = (n % 2).double(), (n // 2 % 4).double()
            v = torch.where(e > 0, (1 + m / 2) * torch.pow(2.0, e - 1), m / 2) * (1 - 2 * (n // 8).double())
            values.append(v * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 1))
        return values[0] @ values[1].t().contiguous() + state["bias"].double()
    if kind == "norm_backward":
        leaves = [state[k].double().requires_grad_() for k in ("x", "gamma", "beta")]
        res = state["residual"].double().requires_grad_() if case["residual"] else None
        # The saved statistics are inputs: x enters through them as the definition has it, their values are those given.
        x, B, G = leaves[0], case["batch"], case["groups"]
        v = x.reshape(B, -1, G, case["C"] // G)
        mean, rstd = (s.double()[:, None, :, None] for s in state["stats"])
        m = v.mean((1, 3), keepdim=True)
        m = m + (mean - m).detach()
        r = -0.5 * rstd ** 3 * (v - m).square().mean((1, 3), keepdim=True)
        r = r + (rstd - r).detach()
        pre = ((v - m) * r).reshape(x.shape) * leaves[1] + leaves[2]
        pre = pre if res is None else pre + res
        wanted = leaves + ([res] if res is not None else [])
        got = torch.autograd.grad(_exact_act(pre, case["act"]), wanted, state["dy"].double())
        return {"dx": got[0], "dgamma": got[1], "dbeta": got[2], "dresidual": got[3] if res is not None else None}
    if kind == "conv":
        v = state["x"][:, ::case["stride"], ::case["stride"]].double()
    else:
        v = _exact_norm(state["x"], state["gamma"], state["beta"], case["groups"])
    if kind == "norm":
        return _exact_act(v if state["residual"] is None else v + state["residual"].double(), case["act"])
    v = _exact_mx4(v if kind == "conv" else _exact_act(v, "relu"))
    w = _exact_mx4(state["weights"].double().reshape(case["C"], case["N"]).t().contiguous())
    y = torch.matmul(v.reshape(-1, case["C"]), w.t().contiguous()).reshape(*v.shape[:-1], case["N"]) + state["bias"].double()
    return _exact_act(y if state["residual"] is None else y + state["residual"].double(), case["act"])
