"""The operators around a pruned network's convolutions, as measurable cases: what a candidate of the pruning loop needs for
its short training and what an accepted one is stored and run with.

``norm``        group norm with an activation (and a shortcut added before it) on channels-last activations
``norm_grad``   its gradients: of the input, the scale, the shift and the shortcut
``clip``        global norm of the gradients of a network's parameters, and clipping to a largest norm
``quantize``    rounding to the 4-bit floating point of the OCP Microscaling formats (blocks of 32 values along the channels that
                share a power of two as their scale); what is returned are the values that the codes stand for
``mx_fc``       product of activations, rounded that way on the way in, with weights kept in that format: fully connected and
                1x1 layers, with bias, shortcut and activation

Activations are channels last: bf16 with the channels padded to ``padded(C)`` (pad lanes zero), float32 without padding.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DEV = "cuda"
BLOCK = 32          # values that share a scale


def padded(C):
    """Channels in memory of a bf16 tensor: a multiple of 8 up to 128 channels, of 16 above."""
    return -(-C // 8) * 8 if C <= 128 else -(-C // 16) * 16


# ---------------------------------------------------------------------------------------------------------------- cases

def _norm(name, batch, hw, C, groups, act, residual=False, dtype="bf16", kind="norm"):
    return {"name": name, "kind": kind, "batch": batch, "hw": hw, "C": C, "groups": groups, "act": act, "residual": residual, "dtype": dtype}


def _fc(name, rows, features, out, act, residual=False, out_f32=False):
    return {"name": name, "kind": "mx_fc", "rows": rows, "in": features, "out": out, "act": act, "residual": residual, "out_f32": out_f32}


def listed():
    return [
        # one image in the last stage of a pruned ResNet-18 (358 filters kept become 352 = 32 groups of 11): latency
        _norm("norm_b1_7x7_c352", 1, 7, 352, 32, "relu", residual=True),
        # float32 activations of a short training, batch 8, an odd number of channels in groups of 13
        _norm("norm_f32_b8_28x28_c91", 8, 28, 91, 7, "silu", dtype="f32"),
        # the stem's output of a pruned network at batch 64: the largest activation of a pass
        _norm("norm_b64_112x112_c44", 64, 112, 44, 4, "relu"),
        # gradients in a middle stage, batch 8
        _norm("norm_grad_b8_14x14_c180", 8, 14, 180, 12, "relu6", kind="norm_grad"),
        # gradients at batch 64 in the widest 56x56 stage of a pruned MobileNetV2, with a shortcut
        _norm("norm_grad_b64_56x56_c108", 64, 56, 108, 12, "silu", residual=True, kind="norm_grad"),
        # the classifier and last stage alone are trained: few, small gradients
        {"name": "clip_12_small", "kind": "clip", "tensors": 12, "total": 90_000, "dtype": "f32", "aligned": True, "max_norm": 1.0},
        # all parameters of a ResNet-18: 62 gradients, 11.7 million values
        {"name": "clip_62_11M", "kind": "clip", "tensors": 62, "total": 11_700_000, "dtype": "f32", "aligned": True, "max_norm": 5.0},
        # the pooled features of one image on their way into a 4-bit classifier
        {"name": "quantize_1x512", "kind": "quantize", "rows": 1, "C": 512, "dtype": "bf16"},
        # a whole activation at batch 64 (56x56 pixels of 108 channels)
        {"name": "quantize_200704x108", "kind": "quantize", "rows": 200_704, "C": 108, "dtype": "bf16"},
        # classifier of one image: 1280 features, 1000 classes, float32 logits
        _fc("mx_fc_1_1280_1000", 1, 1280, 1000, "none", out_f32=True),
        # the first fully connected layer of a VGG-16 for 224x224 images, batch 8
        _fc("mx_fc_8_25088_4096", 8, 25_088, 4096, "relu"),
        # a 1x1 projection at batch 64, 14x14 pixels, with the block's shortcut; 12544 rows
        _fc("mx_fc_12544_960_320", 12_544, 960, 320, "none", residual=True),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST_ELEMENTS = 64 * 112 * 112 * 44        # of an activation
MOST_CLIP = 11_700_000
MOST_FLOPS = 2 * 12_544 * 960 * 320
MOST_QUANTIZE = 200_704 * 108


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "clip", "quantize", "mx_fc", "mx_fc"])
    if kind in ("norm", "norm_grad"):
        most = MOST_ELEMENTS if kind == "norm" else 64 * 56 * 56 * 108
        while True:
            batch, hw, per, groups = _spread(rng, 1, 128), _spread(rng, 1, 112), _spread(rng, 1, 40), _spread(rng, 1, 32)
            dtype, residual = rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.4
            cost = batch * hw * hw * per * groups * (2 if dtype == "f32" else 1) * (1.5 if residual and kind == "norm" else 1)
            if cost <= most and hw * hw * per >= 16:
                break
        return {"kind": kind, "batch": batch, "hw": hw, "C": per * groups, "groups": groups, "act": rng.choice(["none", "relu", "relu6", "silu"]),
                "residual": residual, "dtype": dtype}
    if kind == "clip":
        tensors = _spread(rng, 1, 400)
        dtype = rng.choice(["f32", "f32", "bf16"])
        return {"kind": kind, "tensors": tensors, "total": _spread(rng, max(1000, 4 * tensors), MOST_CLIP), "dtype": dtype,
                "aligned": rng.random() < 0.7, "max_norm": round(10.0 ** rng.uniform(-2, 4), 3)}
    if kind == "quantize":
        C = _spread(rng, 1, 2048)
        return {"kind": kind, "rows": _spread(rng, 1, MOST_QUANTIZE // C), "C": C, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    while True:
        rows, features, out = _spread(rng, 1, 50_176), _spread(rng, 8, 4096), _spread(rng, 8, 4096)
        if 2 * rows * features * out <= MOST_FLOPS and rows * (features + out) <= MOST_QUANTIZE:
            break
    return {"kind": "mx_fc", "rows": rows, "in": features, "out": out, "act": rng.choice(["none", "relu", "relu6"]),
            "residual": rng.random() < 0.4, "out_f32": rng.random() < 0.2}


# ---------------------------------------------------------------------------------------------------------------- inputs

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _lanes(C, dtype):
    return padded(C) if dtype == "bf16" else C


def _activation(g, rows, C, dtype, scale=None, shift=None):
    """Rows of C channels in memory's form: normal values, spread and centred channel by channel as convolutions leave them."""
    lanes = _lanes(C, dtype)
    x = torch.zeros((rows, lanes), dtype=TYPES[dtype], device=DEV)
    v = torch.randn((rows, C), generator=g, device=DEV)
    if scale is not None:
        v.mul_(scale).add_(shift)
    x[:, :C] = v
    return x


def _tensor_sizes(case):
    """Sizes of a network's parameters: shares of the total that span three orders of magnitude, biases among them."""
    n, total = case["tensors"], case["total"]
    shares = [10.0 ** (3.0 * ((7 * i + 3) % n) / max(n - 1, 1)) for i in range(n)]
    s = sum(shares)
    return [max(1, int(total * v / s)) for v in shares]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("norm", "norm_grad"):
        N, hw, C, G = case["batch"], case["hw"], case["C"], case["groups"]
        dtype = case["dtype"]
        scale = torch.exp(0.5 * torch.randn(C, generator=g, device=DEV))
        shift = torch.randn(C, generator=g, device=DEV)
        shape = (N, hw, hw, _lanes(C, dtype))
        s["x"] = _activation(g, N * hw * hw, C, dtype, scale, shift).view(shape)
        s["gamma"] = 1.0 + 0.2 * torch.randn(C, generator=g, device=DEV)
        s["beta"] = 0.2 * torch.randn(C, generator=g, device=DEV)
        s["residual"] = _activation(g, N * hw * hw, C, dtype).view(shape) if case["residual"] else None
        if kind == "norm_grad":
            s["dy"] = _activation(g, N * hw * hw, C, dtype).view(shape)
            v = s["x"][..., :C].double().reshape(N, hw * hw, G, C // G)        # what the forward pass kept
            var, mean = torch.var_mean(v, dim=(1, 3), correction=0)
            s["stats"] = torch.stack([mean, 1.0 / torch.sqrt(var + EPS)], dim=-1).float()
    elif kind == "clip":
        sizes, step = _tensor_sizes(case), 32 if case["aligned"] else 1
        starts, at = [], 0
        for n in sizes:
            starts.append(at)
            at += -(-n // step) * step
        flat = torch.zeros(at, device=DEV)
        for o, n in zip(starts, sizes):
            flat[o:o + n] = torch.randn(n, generator=g, device=DEV) * (0.02 / (1.0 + math.log(n)))
        s["flat"] = flat.to(TYPES[case["dtype"]])
        s["clipped"] = torch.zeros_like(s["flat"])
        s["grads"] = [s["flat"][o:o + n] for o, n in zip(starts, sizes)]
        s["into"] = [s["clipped"][o:o + n] for o, n in zip(starts, sizes)]
    elif kind == "quantize":
        s["x"] = _activation(g, case["rows"], case["C"], case["dtype"], torch.exp(torch.randn(case["C"], generator=g, device=DEV)), 0.0)
    else:
        rows, features, out = case["rows"], case["in"], case["out"]
        s["x"] = torch.zeros((rows, padded(features)), dtype=torch.bfloat16, device=DEV)
        s["x"][:, :features] = torch.randn((rows, features), generator=g, device=DEV).abs_()        # as an activation leaves them
        w = torch.randn((out, features), generator=g, device=DEV) * math.sqrt(2.0 / features)
        s["codes"], s["scales"] = _packed(w)
        s["bias"] = torch.zeros(padded(out), device=DEV)
        s["bias"][:out] = 0.1 * torch.randn(out, generator=g, device=DEV)
        s["residual"] = _activation(g, rows, out, "bf16") if case["residual"] else None
    return s


# ------------------------------------------------------------------------------------------------------- 4-bit values

def _power(exponent):
    """Two to a whole power, as a float64 put together from its bits."""
    return ((exponent.to(torch.int64) + 1023) << 52).view(torch.float64)


def _rounded(x):
    """Rows in blocks of 32: the rounded magnitudes' multiples of the scale, and the scales' exponents.  The scale is
    2^(floor(log2 of the largest magnitude) - 2), not below 2^-127; a block that holds a NaN or an infinity has none (NaN)."""
    rows, C = x.shape
    blocks = -(-C // BLOCK)
    v = torch.zeros((rows, blocks * BLOCK), dtype=torch.float64, device=x.device)
    v[:, :C] = x
    v = v.view(rows, blocks, BLOCK)
    top = v.abs().amax(-1, keepdim=True)
    exponent = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127)
    a = v.abs() * _power(-exponent)
    q = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2))).clamp(max=6)
    q = torch.where(torch.isfinite(top), torch.copysign(q, v), float("nan"))
    return q, exponent


def _packed(w):
    """Weights in memory's form: two codes to a byte, [rows][blocks * 16] (the value with the lower index in the low half), and the
    scales' exponents plus 127 in tiles of 128 rows by 4 blocks, [rows / 128][blocks / 4][row % 32][row / 32 % 4][block % 4]."""
    rows, _ = w.shape
    q, exponent = _rounded(w)
    blocks = q.shape[1]
    a = q.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    code = code.view(rows, blocks * 16, 2)
    tiles = torch.zeros((-(-rows // 128) * 128, -(-blocks // 4) * 4), dtype=torch.uint8, device=w.device)
    tiles[:rows, :blocks] = (exponent[..., 0] + 127).to(torch.uint8)
    tiles = tiles.view(-(-rows // 128), 4, 32, -(-blocks // 4), 4).permute(0, 3, 2, 1, 4).contiguous()
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), tiles


def _unpacked(codes, scales, C):
    """float32 values of packed weights."""
    rows, blocks = codes.shape[0], codes.shape[1] // 16
    code = torch.stack([codes & 15, codes >> 4], dim=-1).view(rows, blocks, BLOCK).to(torch.int32)
    m = code & 7
    a = torch.where(m < 2, 0.5 * m, (1.0 + 0.5 * (m & 1)) * torch.exp2((m >> 1).float() - 1.0))
    q = torch.where(code >= 8, -a, a)
    exponent = scales.permute(0, 3, 2, 1, 4).reshape(scales.shape[0] * 128, -1)[:rows, :blocks].to(torch.int32) - 127
    return (q * _power(exponent).unsqueeze(-1)).float().view(rows, -1)[:, :C]


# ------------------------------------------------------------------------------------------------------------ plain forms

def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "relu6":
        return torch.where(z < 0, 0.0, torch.where(z > 6, 6.0, z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "relu6":
        return ((z > 0) & (z < 6)).to(z.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _stored(v, like):
    """Values of the logical channels in the form of `like`."""
    y = torch.zeros_like(like)
    y[..., :v.shape[-1]] = v
    return y


def _plain_norm(s):
    c = s["case"]
    N, hw, C, G = c["batch"], c["hw"], c["C"], c["groups"]
    x = s["x"][..., :C].float().reshape(N, hw * hw, G, C // G)
    mean = x.mean(dim=(1, 3), keepdim=True)
    var = (x - mean).square().mean(dim=(1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt(var + EPS)
    z = ((x - mean) * rstd).reshape(N, hw, hw, C) * s["gamma"] + s["beta"]
    if s["residual"] is not None:
        z = z + s["residual"][..., :C].float()
    return {"y": _stored(_act(z, c["act"]), s["x"]), "stats": torch.cat([mean, rstd], dim=-1).reshape(N, G, 2)}


def _plain_norm_grad(s):
    c = s["case"]
    N, hw, C, G = c["batch"], c["hw"], c["C"], c["groups"]
    shape = (N, hw * hw, G, C // G)
    mean, rstd = (s["stats"][..., k].reshape(N, 1, G, 1) for k in (0, 1))
    gamma, beta = s["gamma"].view(G, C // G), s["beta"].view(G, C // G)
    x = s["x"][..., :C].reshape(shape)
    # the sides of the borders at 0 and 6 need 64 bits: values next to them take or lose their whole gradient
    z = (x.double() - mean.double()) * rstd.double() * gamma.double() + beta.double()
    if s["residual"] is not None:
        z = z + s["residual"][..., :C].reshape(shape).double()
    dz = s["dy"][..., :C].float().reshape(shape) * _act_slope(z, c["act"]).float()
    xhat = (x.float() - mean) * rstd
    t = dz * gamma
    m1, m2 = t.mean(dim=(1, 3), keepdim=True), (t * xhat).mean(dim=(1, 3), keepdim=True)
    dx = rstd * (t - m1 - xhat * m2)
    got = {"dx": _stored(dx.reshape(N, hw, hw, C), s["x"]), "dgamma": (dz * xhat).sum(dim=(0, 1)).reshape(C), "dbeta": dz.sum(dim=(0, 1)).reshape(C)}
    if s["residual"] is not None:
        got["dresidual"] = _stored(dz.reshape(N, hw, hw, C), s["x"])
    return got


def _plain_clip(s):
    v = s["flat"].float()
    norm = torch.sqrt(v.double().square().sum())
    factor = (s["case"]["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    return {"norm": norm.float().view(1), "clipped": (v * factor).to(s["flat"].dtype)}


def _plain_quantize(s):
    c = s["case"]
    q, exponent = _rounded(s["x"][:, :c["C"]])
    return {"values": _stored((q * _power(exponent)).view(c["rows"], -1)[:, :c["C"]].to(s["x"].dtype), s["x"])}


def _plain_mx_fc(s):
    c = s["case"]
    q, exponent = _rounded(s["x"][:, :c["in"]])
    x = (q * _power(exponent)).float().view(c["rows"], -1)[:, :c["in"]]
    z = x @ _unpacked(s["codes"], s["scales"], c["in"]).t()[:, :c["out"]] + s["bias"][:c["out"]]
    if s["residual"] is not None:
        z = z + s["residual"][:, :c["out"]].float()
    z = _act(z, c["act"])
    if c["out_f32"]:
        return {"y": z}
    y = torch.zeros((c["rows"], padded(c["out"])), dtype=torch.bfloat16, device=z.device)
    y[:, :c["out"]] = z
    return {"y": y}


# ---------------------------------------------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2207_01260_b200 as cp
    c, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        y, stats = cp.cprune_group_norm(s["x"], c["C"], c["groups"], s["gamma"], s["beta"], EPS, c["act"], s["residual"])
        return {"y": y, "stats": stats}
    if kind == "norm_grad":
        dx, dgamma, dbeta, dres = cp.cprune_group_norm_backward(s["dy"], s["x"], c["C"], c["groups"], s["stats"], s["gamma"], s["beta"], c["act"],
                                                                s["residual"])
        got = {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        if dres is not None:
            got["dresidual"] = dres
        return got
    if kind == "clip":
        norm = cp.cprune_clip_gradients(s["grads"], c["max_norm"], out=s["into"])
        return {"norm": norm, "clipped": s["clipped"]}
    if kind == "quantize":
        return {"values": cp.cprune_mx_quantize(s["x"], c["C"], values=True)[2]}
    return {"y": cp.cprune_mx_fc(s["x"], c["in"], s["codes"], s["scales"], s["bias"], c["out"], c["act"], s["residual"], out_f32=c["out_f32"])}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip, "quantize": _plain_quantize, "mx_fc": _plain_mx_fc}[state["case"]["kind"]](state)


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n = case["batch"] * case["hw"] ** 2 * case["C"]
        size = 2 if case["dtype"] == "bf16" else 4
        tensors = (2 if kind == "norm" else 3) + (1 if case["residual"] else 0) + (1 if case["residual"] and kind == "norm_grad" else 0)
        return {"bytes": n * size * tensors + 16 * case["C"] + 8 * case["batch"] * case["groups"], "flops": n * (10 if kind == "norm" else 20)}
    if kind == "clip":
        n = sum(_tensor_sizes(case))
        return {"bytes": 2 * n * (2 if case["dtype"] == "bf16" else 4) + 4, "flops": 3 * n}
    if kind == "quantize":
        n = case["rows"] * case["C"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * size * 2 + n * 17 / 32, "flops": 4 * n}
    rows, features, out = case["rows"], case["in"], case["out"]
    return {"bytes": 2 * rows * features + out * features * 17 / 32 + 4 * out + rows * out * ((4 if case["out_f32"] else 2) + (2 if case["residual"] else 0)),
            "flops": 2.0 * rows * features * out}


# ------------------------------------------------------------------------------------------------------- 64-bit definitions

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(x):
    """Values of the format nearest to a matrix's, by comparison with every one of them (ties: the even code)."""
    rows, C = x.shape
    got = torch.empty_like(x)
    table = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)          # even codes first, so that they win a tie
    for at in range(0, C, BLOCK):
        v = x[:, at:at + BLOCK]
        top = v.abs().max(dim=1, keepdim=True).values
        scale = torch.exp2((torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2).clamp(min=-127.0))
        # a logarithm rounded to the wrong side of a whole number is put right: 4 <= top / scale < 8, but for the smallest scale
        scale = torch.where((scale > 2.0 ** -127) & (scale * 4 > top), scale / 2, torch.where(scale * 8 <= top, scale * 2, scale))
        best, distance = None, None
        for k in order:
            d = (v.abs() - table[k] * scale).abs()
            if best is None:
                best, distance = (table[k] * scale).expand_as(v), d
            else:
                best, distance = torch.where(d < distance, table[k] * scale, best), torch.minimum(d, distance)
        got[:, at:at + BLOCK] = torch.where(torch.isfinite(top), torch.where(v < 0, -best, best), float("nan"))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    kind, d = case["kind"], torch.float64

    def lanes(v, dtype):
        return torch.nn.functional.pad(v, (0, _lanes(v.shape[-1], dtype) - v.shape[-1]))

    def slope(z):
        z = z.detach().requires_grad_(True)
        a = case["act"]
        y = {"none": lambda: z * 1.0, "relu": lambda: torch.relu(z), "relu6": lambda: torch.nn.functional.relu6(z),
             "silu": lambda: torch.nn.functional.silu(z)}[a]()
        return y.detach(), torch.autograd.grad(y.sum(), z)[0]

    if kind in ("norm", "norm_grad"):
        N, hw, C, G = case["batch"], case["hw"], case["C"], case["groups"]
        dt = case["dtype"]
        x = s["x"][..., :C].to(d)
        x = x.permute(0, 3, 1, 2).reshape(N, G, -1)                    # channels first: a group is one run of values
        gamma, beta = (v.to(d).view(1, C, 1) for v in (s["gamma"], s["beta"]))
        if kind == "norm":
            var, mean = torch.var_mean(x, dim=2, correction=0, keepdim=True)
            rstd = (var + EPS).rsqrt()
        else:
            mean, rstd = s["stats"][..., :1].to(d), s["stats"][..., 1:].to(d)
        xhat = ((x - mean) * rstd).reshape(N, C, hw * hw)
        del x
        z = xhat * gamma + beta
        if s["residual"] is not None:
            z = z + s["residual"][..., :C].to(d).permute(0, 3, 1, 2).reshape(N, C, hw * hw)
        back = lambda v: lanes(v.reshape(N, C, hw, hw).permute(0, 2, 3, 1), dt).contiguous()  # noqa: E731
        y, f = slope(z)
        del z
        if kind == "norm":
            return {"y": back(y), "stats": torch.cat([mean, rstd], dim=2)}
        del y
        dz = s["dy"][..., :C].to(d).permute(0, 3, 1, 2).reshape(N, C, hw * hw) * f
        got = {"dgamma": (dz * xhat).sum(dim=(0, 2)), "dbeta": dz.sum(dim=(0, 2))}
        if s["residual"] is not None:
            got["dresidual"] = back(dz)
        t, h = (dz * gamma).reshape(N, G, -1), xhat.reshape(N, G, -1)
        got["dx"] = back(rstd * (t - t.mean(2, keepdim=True) - h * (t * h).mean(2, keepdim=True)))
        return got
    if kind == "clip":
        v = torch.cat([t.to(d) for t in s["grads"]])
        norm = torch.linalg.vector_norm(v)
        return {"norm": norm.view(1), "clipped": s["flat"].to(d) * min(1.0, case["max_norm"] / (float(norm) + 1e-6))}
    if kind == "quantize":
        return {"values": lanes(_nearest(s["x"][:, :case["C"]].to(d)), case["dtype"])}
    rows, features, out = case["rows"], case["in"], case["out"]
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=d, device=DEV)
    w = torch.empty((out, features), dtype=d, device=DEV)
    r = torch.arange(out, device=DEV)
    for k in range(features):
        byte = s["codes"][:, k // 2].long()
        e = s["scales"][r // 128, k // 128, r % 32, r // 32 % 4, k // 32 % 4].to(d)
        w[:, k] = table[(byte >> 4) if k % 2 else (byte & 15)] * torch.exp2(e - 127)
    z = torch.nn.functional.linear(_nearest(s["x"][:, :features].to(d)), w, s["bias"][:out].to(d))
    if s["residual"] is not None:
        z = z + s["residual"][:, :out].to(d)
    y = slope(z)[0]
    return {"y": y if case["out_f32"] else lanes(y, "bf16")}
