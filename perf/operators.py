"""The operators around the pruned convolutions whose speed matters here: group normalisation with an
activation (channels last, forward and backward), microscaled 4-bit floating point (MXFP4: quantisation,
and the linear layer on quantised weights), and the change of channel order that joins them to the NCHW
convolutions.

A case is a dict of plain values; ``op`` says which operator:

``reorder``   ``n`` images, ``c`` channels, ``h`` x ``w`` pixels; ``to`` "last" or "first"; types ``src``, ``dst``
``norm``      ``n``, ``h``, ``w``, ``c``, ``groups``, ``act``, ``dtype``; ``wide``: channels of the tensor that x is
              the first ``c`` of (a slice of a wider one); forward, with the statistics
``norm_bwd``  the same, backward: dx, dgamma, dbeta from dy, x and the forward's statistics
``quantise``  ``rows`` x ``cols`` values of ``dtype`` to MXFP4, and the values that they stand for back
``linear``    ``rows`` x ``k`` activations of ``dtype`` times ``out`` x ``k`` MXFP4 weights, bias and ``act``;
              ``quantised``: the activations are MXFP4 already; output of type ``dst``

``own`` false: the plain forms; true: the framework's operators.
"""

import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # one frame: a 3x3 layer's fp32 output goes on to a pointwise layer
        {"name": "reorder_frame", "op": "reorder", "n": 1, "c": 256, "h": 56, "w": 56, "to": "last", "src": "f32", "dst": "bf16"},
        # a batch of pointwise outputs goes back to the 3x3 layers, at sizes that are no multiples of anything
        {"name": "reorder_ragged", "op": "reorder", "n": 48, "c": 203, "h": 61, "w": 45, "to": "first", "src": "f16", "dst": "f32"},
        # the last stage of a network on one image: the smallest call, where latency counts
        {"name": "norm_frame", "op": "norm", "n": 1, "h": 7, "w": 7, "c": 512, "groups": 32, "act": "relu", "dtype": "f32", "wide": 512},
        # the first stage of a network on a batch
        {"name": "norm_batch", "op": "norm", "n": 64, "h": 56, "w": 56, "c": 256, "groups": 32, "act": "silu", "dtype": "f16", "wide": 256},
        # a training step on a few odd images, three channels a group, x a slice of a wider tensor
        {"name": "norm_bwd_ragged", "op": "norm_bwd", "n": 6, "h": 45, "w": 61, "c": 96, "groups": 32, "act": "relu", "dtype": "f32", "wide": 160},
        # a training step on a batch
        {"name": "norm_bwd_batch", "op": "norm_bwd", "n": 64, "h": 56, "w": 56, "c": 256, "groups": 32, "act": "silu", "dtype": "bf16", "wide": 256},
        # the flattened features of one image
        {"name": "quantise_row", "op": "quantise", "rows": 1, "cols": 25088, "dtype": "f32"},
        # the pixels of a batch before a pointwise layer
        {"name": "quantise_batch", "op": "quantise", "rows": 200704, "cols": 256, "dtype": "f16"},
        # the first fully connected layer of a classifier, one image served: the weights' bytes count
        {"name": "linear_row", "op": "linear", "rows": 1, "k": 25088, "out": 4096, "act": "relu", "dtype": "f16", "dst": "f16", "quantised": False},
        # the last one, odd sizes, a few images
        {"name": "linear_ragged", "op": "linear", "rows": 77, "k": 4100, "out": 1000, "act": "none", "dtype": "f32", "dst": "f32", "quantised": False},
        # a pointwise layer on the pixels of a batch
        {"name": "linear_pixels", "op": "linear", "rows": 50176, "k": 128, "out": 512, "act": "silu", "dtype": "f16", "dst": "f16", "quantised": False},
        # a large product, activations quantised before (two layers read them): the largest case
        {"name": "linear_large", "op": "linear", "rows": 8192, "k": 8192, "out": 8192, "act": "none", "dtype": "bf16", "dst": "bf16", "quantised": True},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high, most):
    """A size of [low, min(high, most)], even in its logarithm; two in five are rounded up to a multiple of 16."""
    high = max(low, min(high, int(most)))
    v = _log(rng, low, high)
    return min(high, (v + 15) // 16 * 16) if rng.random() < 0.4 else v


def draw(rng):
    op = rng.choice(["reorder", "norm", "norm", "norm_bwd", "norm_bwd", "quantise", "linear", "linear", "linear"])
    kind = lambda: rng.choice(["f32", "f16", "bf16"])  # noqa: E731
    act = rng.choice(["none", "relu", "silu"])
    if op in ("reorder", "norm", "norm_bwd"):
        n = _log(rng, 1, 64)
        h = _log(rng, 7, 112)
        w = max(5, min(112, int(h * rng.uniform(0.7, 1.4))))
        most = 6e7 / (n * h * w)
    if op == "reorder":
        return {"op": op, "n": n, "c": _size(rng, 3, 960, most), "h": h, "w": w, "to": rng.choice(["last", "first"]), "src": kind(), "dst": kind()}
    if op in ("norm", "norm_bwd"):
        groups = rng.choice([1, 4, 8, 16, 32, 32, 32])
        per = _log(rng, 1, max(1, min(960 // groups, int(most / groups))))
        wide = groups * per + rng.choice([0, 0, 0, 5, 64])
        return {"op": op, "n": n, "h": h, "w": w, "c": groups * per, "groups": groups, "act": act, "dtype": kind(), "wide": wide}
    if op == "quantise":
        cols = _size(rng, 24, 25088, 25088)
        return {"op": op, "rows": _log(rng, 1, max(1, min(200704, int(5e7 / cols)))), "cols": cols, "dtype": kind()}
    k, out = _size(rng, 48, 25088, 25088), _size(rng, 16, 8192, 8192)
    rows = _log(rng, 1, max(1, min(50176, int(4e11 / (k * out)), int(1e8 / max(k, out)))))
    quantised = rng.random() < 0.3
    return {"op": op, "rows": rows, "k": k, "out": out, "act": act, "dtype": kind(), "dst": kind(), "quantised": quantised}


# -- the values that programs have in hand ------------------------------------------------------------

def _random(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _pack(values, scales):
    """(values on the grid of 4 bits, exponents) of whole blocks -> stored codes and scales."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=values.device)
    code = torch.bucketize(values.abs(), grid).to(torch.uint8) + 8 * torch.signbit(values).to(torch.uint8)
    code = code.reshape(code.shape[0], -1)
    return code[:, 0::2] + 16 * code[:, 1::2], scales


def _stored(x):
    """x [rows][cols] -> MXFP4 as it is kept: codes [rows][ceil(cols/128)*64], scales [rows][ceil(cols/128)*4]."""
    codes, scales = [], []
    step = max(1, (1 << 25) // max(1, x.shape[1]))
    for i in range(0, x.shape[0], step):
        c, s = _pack(*_quantised(x[i:i + step]))
        codes.append(c)
        scales.append(s)
    return torch.cat(codes), torch.cat(scales)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    state = {"case": case}
    if op == "reorder":
        shape = (case["n"], case["c"], case["h"], case["w"]) if case["to"] == "last" else (case["n"], case["h"], case["w"], case["c"])
        state["x"] = _random(g, *shape).to(TYPES[case["src"]])
        there = shape[:1] + (shape[2:] + shape[1:2] if case["to"] == "last" else shape[3:] + shape[1:3])
        state["out"] = torch.empty(there, dtype=TYPES[case["dst"]], device="cuda")
    elif op in ("norm", "norm_bwd"):
        n, h, w, c, wide = (case[k] for k in ("n", "h", "w", "c", "wide"))
        # channels differ in level and spread, as behind a convolution
        level, spread = _random(g, wide), torch.exp(0.5 * _random(g, wide))
        x = (_random(g, n, h, w, wide) * spread + level).to(TYPES[case["dtype"]])[..., :c]
        state.update(x=x, gamma=1 + 0.3 * _random(g, c), beta=0.3 * _random(g, c))
        state["out"] = torch.empty((n, h, w, c), dtype=x.dtype, device="cuda")
        if op == "norm_bwd":
            state["dy"] = _random(g, n, h, w, c).to(x.dtype)
            # what the forward pass kept
            v = x.float().reshape(n, h * w, case["groups"], -1)
            var, mean = torch.var_mean(v, dim=(1, 3), unbiased=False)
            state.update(mean=mean.contiguous(), rstd=torch.rsqrt(var + EPS).contiguous())
    elif op == "quantise":
        x = _random(g, case["rows"], case["cols"])
        x *= torch.exp(0.5 * _random(g, case["cols"]))
        state["x"] = torch.relu(x).to(TYPES[case["dtype"]]) if seed % 2 else x.to(TYPES[case["dtype"]])
        state["out"] = torch.empty_like(state["x"])
        pieces = -(-case["cols"] // 128)
        state["codes"], state["scales"] = (torch.empty((case["rows"], pieces * b), dtype=torch.uint8, device="cuda") for b in (64, 4))
    else:
        rows, k, out = case["rows"], case["k"], case["out"]
        x = (_random(g, rows, k) * torch.exp(0.3 * _random(g, k))).to(TYPES[case["dtype"]])
        state["w"], state["w_scales"] = _stored(_random(g, out, k) * math.sqrt(2 / k))
        state["bias"] = 0.1 * _random(g, out)
        state["x"], state["x_scales"] = _stored(x) if case["quantised"] else (x, None)
        state["out"] = torch.empty((rows, out), dtype=TYPES[case["dst"]], device="cuda")
    return state


# -- the plain forms ----------------------------------------------------------------------------------

def _quantised(x):
    """x [rows][cols] -> values on the grid of 4 bits [rows][blocks][32], and the scales' bytes [rows][blocks]."""
    x = x.float()
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 128)).reshape(x.shape[0], -1, 32)
    most = x.abs().amax(dim=2)
    e = (torch.frexp(most).exponent - 3).clamp(-127, 127)
    e = torch.where(most == 0, -127, e)
    a = torch.ldexp(x, -e.unsqueeze(2))
    m = a.abs()
    q = torch.where(m < 2, torch.round(m * 2) / 2, torch.where(m < 4, torch.round(m), torch.round(m / 2) * 2)).clamp(max=6)
    fine = torch.isfinite(most)
    q = torch.copysign(torch.where(fine.unsqueeze(2), q, 0.0), x)
    return q, torch.where(fine, e + 127, 255).to(torch.uint8)


def _values(q, scales):
    """What values on the grid and scales' bytes stand for, [rows][padded cols]."""
    v = torch.ldexp(q, scales.to(torch.int32).unsqueeze(2) - 127)
    return torch.where(scales.unsqueeze(2) == 255, float("nan"), v).reshape(q.shape[0], -1)


def _unpacked(codes):
    """Stored codes -> values on the grid [rows][blocks][32]."""
    both = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1, 32)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    return grid[both.to(torch.int32)]


def _activated(z, act):
    return torch.relu(z) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def _plain(state):
    case = state["case"]
    op = case["op"]
    x = state["x"]
    if op == "reorder":
        return x.permute((0, 2, 3, 1) if case["to"] == "last" else (0, 3, 1, 2)).to(TYPES[case["dst"]]).contiguous()
    if op in ("norm", "norm_bwd"):
        n, h, w, c = x.shape
        v = x.float().reshape(n, h * w, case["groups"], c // case["groups"])
        gamma, beta = (state[k].reshape(1, 1, case["groups"], -1) for k in ("gamma", "beta"))
    if op == "norm":
        mean = v.mean(dim=(1, 3), keepdim=True)
        d = v - mean
        rstd = torch.rsqrt((d * d).mean(dim=(1, 3), keepdim=True) + EPS)
        y = _activated(d * rstd * gamma + beta, case["act"])
        return y.reshape(n, h, w, c).to(x.dtype), mean.reshape(n, -1), rstd.reshape(n, -1)
    if op == "norm_bwd":
        mean, rstd = (state[k].reshape(n, 1, -1, 1) for k in ("mean", "rstd"))
        xh = (v - mean) * rstd
        dz = state["dy"].float().reshape(v.shape)
        if case["act"] != "none":
            z = xh * gamma + beta
            if case["act"] == "relu":
                dz = dz * (z > 0)
            else:
                s = torch.sigmoid(z)
                dz = dz * (s * (1 + z * (1 - s)))
        dbeta, dgamma = dz.sum(dim=(0, 1)), (dz * xh).sum(dim=(0, 1))
        dz = dz * gamma
        a, b = dz.mean(dim=(1, 3), keepdim=True), (dz * xh).mean(dim=(1, 3), keepdim=True)
        dx = rstd * (dz - a - xh * b)
        return dx.reshape(n, h, w, c).to(x.dtype), dgamma.reshape(c), dbeta.reshape(c)
    if op == "quantise":
        return _values(*_quantised(x))[:, :case["cols"]].to(x.dtype)
    a = _values(_unpacked(x), state["x_scales"]) if case["quantised"] else _values(*_quantised(x))
    b = _values(_unpacked(state["w"]), state["w_scales"])
    return _activated(torch.addmm(state["bias"], a, b.t()), case["act"]).to(TYPES[case["dst"]])


def run(state):
    if not own:
        return _plain(state)
    from paper_2001_00138_amd import binding as B
    case = state["case"]
    op = case["op"]
    if op == "reorder":
        reorder = B.patdnn_channels_last if case["to"] == "last" else B.patdnn_channels_first
        return reorder(state["x"], state["out"])
    if op == "norm":
        return B.patdnn_group_norm(state["x"], case["groups"], state["gamma"], state["beta"], state["out"], eps=EPS, act=case["act"])
    if op == "norm_bwd":
        return B.patdnn_group_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], case["groups"], state["gamma"], state["beta"],
                                            state["out"], act=case["act"])
    if op == "quantise":
        codes, scales = B.patdnn_mxfp4_quantize(state["x"], state["codes"], state["scales"])
        return B.patdnn_mxfp4_dequantize(codes, scales, case["cols"], state["out"])
    return B.patdnn_mxfp4_linear(state["x"], state["w"], state["w_scales"], state["bias"], state["out"], x_scales=state["x_scales"], act=case["act"])


# -- the definitions in 64 bits, written apart from the plain forms ------------------------------------

def _exact_values(x):
    """The MXFP4 values of x [rows][cols], by comparing with the midpoints between neighbours of the grid."""
    rows, cols = x.shape
    v = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    v = v.view(rows, -1, 32)
    most = v.abs().max(dim=2, keepdim=True).values
    e = torch.floor(torch.log2(most.clamp(min=2.0 ** -125))) - 2
    # log2 near a power of two may round across it
    e = torch.where(torch.exp2(e + 3) <= most, e + 1, torch.where(torch.exp2(e + 2) > most.clamp(min=2.0 ** -125), e - 1, e))
    unit = torch.exp2(e.clamp(min=-127))
    m = v.abs() / unit
    q = 0.5 * ((m > 0.25).double() + (m >= 0.75) + (m > 1.25) + (m >= 1.75)) + (m > 2.5) + (m >= 3.5) + 2 * (m > 5).double()
    return (q * v.sign() * unit).view(rows, -1)[:, :cols]


def _exact_stored(codes, scales, cols):
    out = torch.zeros((codes.shape[0], codes.shape[1], 2), dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = ((codes >> (4 * half)) & 15).to(torch.int64)
        e, m = (c >> 1) & 3, c & 1
        size = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2((e - 1).double()))
        out[:, :, half] = torch.where(c >= 8, -size, size)
    unit = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)
    return (out.view(codes.shape[0], -1) * unit)[:, :cols]


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    x = state["x"]
    if op == "reorder":
        x = x.double()
        return (x.flatten(2).transpose(1, 2) if case["to"] == "last" else x.flatten(1, 2).transpose(1, 2)).reshape(state["out"].shape)
    if op == "quantise":
        return _exact_values(x)
    if op == "linear":
        out = torch.empty(state["out"].shape, dtype=torch.float64, device=x.device)
        a = _exact_stored(x, state["x_scales"], case["k"]) if case["quantised"] else _exact_values(x)
        for i in range(0, case["out"], 1024):
            b = _exact_stored(state["w"][i:i + 1024], state["w_scales"][i:i + 1024], case["k"])
            out[:, i:i + 1024] = a @ b.t().contiguous() + state["bias"][i:i + 1024].double()
    if op != "linear":
        n, c, groups = case["n"], case["c"], case["groups"]
        gamma, beta = state["gamma"].double(), state["beta"].double()
        spread = lambda t: t.repeat_interleave(c // groups, dim=1).view(n, 1, 1, c)  # noqa: E731
        # images one by one: 64-bit copies of a whole batch would not fit three times
        total = lambda t: torch.stack([u.double().sum(dim=(0, 1)).view(groups, -1).sum(dim=1) for u in t])  # noqa: E731
        count = case["h"] * case["w"] * (c // groups)
        if op == "norm":
            mean = total(x) / count
            square = torch.stack([(u.double() - m).square().sum(dim=(0, 1)).view(groups, -1).sum(dim=1) for u, m in zip(x, spread(mean))])
            rstd = (square / count + EPS) ** -0.5
            out = (x.double() - spread(mean)) * spread(rstd) * gamma + beta
        else:
            mean, rstd = spread(state["mean"].double()), spread(state["rstd"].double())
            dx, dgamma, dbeta = torch.empty(state["dy"].shape, dtype=torch.float64, device=x.device), 0, 0
            for i in range(n):
                xh = (x[i].double() - mean[i]) * rstd[i]
                z = xh * gamma + beta
                s = 1 / (1 + torch.exp(-z))
                slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": s + z * s * (1 - s)}[case["act"]]
                dz = state["dy"][i].double() * slope
                dbeta, dgamma = dbeta + dz.sum(dim=(0, 1)), dgamma + (dz * xh).sum(dim=(0, 1))
                dz = dz * gamma
                per = lambda t: (t.sum(dim=(0, 1)).view(groups, -1).sum(dim=1) / count).repeat_interleave(c // groups)  # noqa: E731
                dx[i] = rstd[i] * (dz - per(dz) - xh * per(dz * xh))
            return dx, dgamma, dbeta
    if case["act"] == "relu":
        out = torch.where(out > 0, out, 0.0)
    elif case["act"] == "silu":
        out = out / (1 + torch.exp(-out))
    return (out, mean, rstd) if op == "norm" else out


def work(case):
    op = case["op"]
    if op == "reorder":
        count = case["n"] * case["c"] * case["h"] * case["w"]
        return {"bytes": count * (BYTES[case["src"]] + BYTES[case["dst"]]), "flops": 0}
    if op in ("norm", "norm_bwd"):
        count, t = case["n"] * case["h"] * case["w"] * case["c"], BYTES[case["dtype"]]
        small = 8 * case["n"] * case["groups"] + 8 * case["c"]
        extra = {"none": 0, "relu": 1, "silu": 4}[case["act"]]
        if op == "norm":
            return {"bytes": 2 * count * t + small, "flops": count * (7 + extra)}
        return {"bytes": 3 * count * t + small + 8 * case["c"], "flops": count * (16 + 2 * extra)}
    if op == "quantise":
        count = case["rows"] * case["cols"]
        return {"bytes": 2 * count * BYTES[case["dtype"]] + 2 * count * 17 / 32, "flops": 3 * count}
    m, k, n = case["rows"], case["k"], case["out"]
    x = m * k * (17 / 32 if case["quantised"] else BYTES[case["dtype"]])
    return {"bytes": x + n * k * 17 / 32 + 4 * n + m * n * BYTES[case["dst"]], "flops": 2 * m * n * k}
