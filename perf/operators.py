"""The operators around the Gated MLP that a training or serving program calls:
the training step of the block (the forward pass that keeps what its gradients
need, and the backward pass), the norms between two blocks with their gate and
residual scale and their backward pass, and products with 4-bit weights for
decoding.

A case is a dict of plain values; "op" is one of

    train_forward   y, and G = X Wg, U = X Wu for the backward pass
    train_backward  the gradients of X and the three weights from that of y
    norm            r = res_scale res + gate * post(y), xn = RMSNorm(r) w_pre
    norm_backward   its gradients
    w4_forward      the whole MLP with 4-bit weights
    w4_matmul       one product with a 4-bit weight

`run` computes a case in plain 32-bit torch operations, or with `own` true by
the library's entry points.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BETA = 1.702  # the swish slope of the SwiGLU variant
EPS = 1e-6
LARGEST = (4096, 4096, 14336)  # T, D, F of the largest listed case


# ---- cases ---------------------------------------------------------------------


def _mlp(name, op, T, D, F, activation="silu"):
    return {"name": name, "op": op, "T": T, "D": D, "F": F, "activation": activation}


def _norm(name, op, T, D, res="bf16", post=True, gate="channel", res_scale=1.0):
    return {"name": name, "op": op, "T": T, "D": D, "res": res, "post": post, "gate": gate, "res_scale": res_scale}


def _w4(name, op, T, D, F, group, zeros=False, activation="silu"):
    return {"name": name, "op": op, "T": T, "D": D, "F": F, "group": group, "zeros": zeros, "activation": activation}


def listed():
    return [
        # One training micro-batch of 4096 tokens on an 8B-class layer, forward ...
        _mlp("train_forward_4096", "train_forward", *LARGEST),
        # ... a short ragged sequence of a small model with the GLU gate.
        _mlp("train_forward_300_glu", "train_forward", 300, 2048, 8192, "sigmoid"),
        # The smallest backward pass: a toy layer, bound by launches.
        _mlp("backward_16_tiny", "train_backward", 16, 256, 512, "swish"),
        # Fine-tuning on one ragged sequence of a 13B-class layer: bound by the
        # weights read and the weight gradients written.
        _mlp("backward_300", "train_backward", 300, 5120, 13824),
        # The backward pass of the micro-batch: bound by the matrix cores.
        _mlp("backward_4096", "train_backward", *LARGEST),
        # Between two blocks while decoding one sequence: bound by latency.
        _norm("norm_decode", "norm", 1, 4096),
        # Between two blocks in training or prefill.
        _norm("norm_4096", "norm", 4096, 4096),
        # An odd width, a residual stream in fp32 and a gate for every token.
        _norm("norm_backward_1000", "norm_backward", 1000, 2056, res="fp32", gate="token", res_scale=0.5),
        # The gradients of norm_4096.
        _norm("norm_backward_4096", "norm_backward", 4096, 4096),
        # Single-stream decode of the 8B-class layer with 4-bit weights.
        _w4("w4_decode", "w4_forward", 1, 4096, 14336, 128),
        # Five sequences, a 13B-class down projection with zero points.
        _w4("w4_matmul_5_zeros", "w4_matmul", 5, 5120, 13824, 64, zeros=True),
        # A small model's batched decode, an odd batch, short groups.
        _w4("w4_batch_33", "w4_forward", 33, 2048, 8192, 32, activation="swish"),
    ]


# (D, F) of the repository's workloads and tests, and of the same class.
_WIDTHS = [(256, 512), (1024, 4096), (1032, 2056), (2048, 8192), (4096, 11008), (4096, 12288), (4096, 14336),
           (4096, 16384), (5120, 13824), (8192, 28672)]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _widths(rng):
    D, F = rng.choice(_WIDTHS)
    if rng.random() < 0.4:  # widths of no particular class
        D = 8 * _log_uniform(rng, 32, 1024)
        F = 8 * max(64, min(3584, int(D / 8 * rng.uniform(2.0, 4.0))))
    return D, F


def draw(rng: random.Random):
    most = work(_mlp("", "train_backward", *LARGEST))
    while True:
        op = rng.choice(["train_forward", "train_backward", "norm", "norm_backward", "w4_forward", "w4_matmul"])
        if op.startswith("train"):
            D, F = _widths(rng)
            c = _mlp("", op, _log_uniform(rng, 1, 4096), D, F, rng.choice(["silu", "silu", "swish", "sigmoid"]))
        elif op.startswith("norm"):
            D = 8 * _log_uniform(rng, 32, 1024)
            c = _norm("", op, _log_uniform(rng, 1, 8192), D, rng.choice(["bf16", "bf16", "fp32"]),
                      rng.random() < 0.7, rng.choice(["none", "channel", "token"]), rng.choice([1.0, 1.0, 0.5]))
        else:
            D, F = _widths(rng)
            c = _w4("", op, _log_uniform(rng, 1, 64), D, F, rng.choice([32, 64, 128, 128]), rng.random() < 0.4,
                    rng.choice(["silu", "silu", "swish", "sigmoid"]))
        del c["name"]
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"]:
            return c


def _groups(case):
    """(rows, columns) of every 4-bit weight of a case, in the order of the call."""
    D, F = case["D"], case["F"]
    return [(D, F), (D, F), (F, D)] if case["op"] == "w4_forward" else [(F, D)]


def work(case):
    op, T, D = case["op"], case["T"], case["D"]
    if op == "norm":
        # y, res and the token gates in, r and xn out; two sums of squares,
        # the scaled sum and two products with gains.
        b = 2 if case["res"] == "bf16" else 4
        return {"bytes": T * D * (2.0 + 2 * b + 2 + (2 if case["gate"] == "token" else 0)), "flops": 10.0 * T * D}
    if op == "norm_backward":
        b = 2 if case["res"] == "bf16" else 4
        # dxn, dr, y and r in, dy and dres out; a token gate in and its gradient out.
        return {"bytes": T * D * (2.0 + b + 2 + b + 2 + b + (4 if case["gate"] == "token" else 0)),
                "flops": 24.0 * T * D}
    F = case["F"]
    if op == "train_forward":
        return {"bytes": 2.0 * (3 * D * F + 2 * T * D + 2 * T * F), "flops": 6.0 * T * D * F}
    if op == "train_backward":
        return {"bytes": 2.0 * (6 * D * F + 3 * T * D + 2 * T * F), "flops": 12.0 * T * D * F}
    nbytes = flops = 0.0
    for K, N in _groups(case):
        groups = -(-K // case["group"])
        nbytes += K * N / 2 + groups * N * (2.5 if case["zeros"] else 2.0)
        flops += 2.0 * T * K * N
    nbytes += 2.0 * T * (2 * D if op == "w4_forward" else F + D)
    return {"bytes": nbytes, "flops": flops}


# ---- inputs --------------------------------------------------------------------


def _normal(gen, rows, cols, scale=1.0, mean=0.0, dtype=torch.bfloat16):
    t = torch.empty((rows, cols), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // cols)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        t[r:r + n] = torch.randn((n, cols), generator=gen, device="cuda") * scale + mean
    return t


def _quantised(gen, K, N, group, zeros):
    """q [K, N] in 0..15, scales [groups, N] bf16 and zero points [groups, N]
    (8 without) of a weight N(0, 1/K), rounded to nearest group by group; the
    last group may be short."""
    groups = -(-K // group)
    w = torch.zeros((groups * group, N), device="cuda")
    w[:K] = torch.randn((K, N), generator=gen, device="cuda") * K ** -0.5
    w = w.view(groups, group, N)
    if zeros:
        low, high = w.amin(1).clamp(max=0), w.amax(1).clamp(min=0)
        s = ((high - low) / 15).clamp(min=1e-8).to(torch.bfloat16)
        z = (-low / s.float()).round().clamp(0, 15).to(torch.uint8)
    else:
        s = (w.abs().amax(1) / 7).clamp(min=1e-8).to(torch.bfloat16)
        z = torch.full((groups, N), 8, dtype=torch.uint8, device="cuda")
    q = (w / s.float()[:, None] + z[:, None]).round().clamp(0, 15).to(torch.uint8)
    return q.view(groups * group, N)[:K].contiguous(), s, z


def _inputs(case, seed):
    """Inputs with the distributions of the repository's generator:
    activations N(0, 1), weights N(0, 1/fan_in); G and U, products of such, are
    N(0, 1) as well.  Gains and channel gates are around 1."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, T, D = case["op"], case["T"], case["D"]
    if op.startswith("norm"):
        res = torch.bfloat16 if case["res"] == "bf16" else torch.float32
        t = {"y": _normal(gen, T, D), "w_pre": _normal(gen, 1, D, 0.2, 1.0)[0], "w_post": None, "gate": None}
        if case["post"]:
            t["w_post"] = _normal(gen, 1, D, 0.2, 1.0)[0]
        if case["gate"] == "channel":
            t["gate"] = _normal(gen, 1, D, 0.2, 0.8)[0]
        if case["gate"] == "token":
            t["gate"] = _normal(gen, T, D, 0.5, 0.5)
        if op == "norm":
            t["res"] = _normal(gen, T, D, 2.0, dtype=res)
        else:
            t.update(r=_normal(gen, T, D, 2.0, dtype=res), dxn=_normal(gen, T, D), dr=_normal(gen, T, D, dtype=res))
        return t
    F = case["F"]
    if op.startswith("train"):
        t = {"x": _normal(gen, T, D), "wg": _normal(gen, D, F, D ** -0.5), "wu": _normal(gen, D, F, D ** -0.5),
             "wd": _normal(gen, F, D, F ** -0.5)}
        if op == "train_backward":
            t.update(g=_normal(gen, T, F), u=_normal(gen, T, F), dy=_normal(gen, T, D))
        return t
    return {"x": _normal(gen, T, _groups(case)[0][0]),
            "w": [_quantised(gen, K, N, case["group"], case["zeros"]) for K, N in _groups(case)]}


def _activation(case):
    kw = {"activation": case["activation"]}
    if case["activation"] == "swish":
        kw["beta"] = BETA
    return kw


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2606_26344_amd import block_norm, train, w4

        op, T, D = case["op"], case["T"], case["D"]
        if op.startswith("train"):
            s["workspace"] = train.make_workspace(T, D, case["F"])
        elif op == "norm_backward":
            s["workspace"] = block_norm.make_workspace(T, D)
        elif op.startswith("w4"):
            # The weights as a serving program holds them: laid out once.
            s["w"] = [w4.pack(q, scale, zero if case["zeros"] else None, group=case["group"])
                      for q, scale, zero in s["w"]]
            s["workspace"] = w4.make_workspace(T, D, case["F"])
    return s


# ---- the library's calls ---------------------------------------------------------


def _run_own(s):
    from paper_2606_26344_amd import block_norm, train, w4

    case = s["case"]
    op = case["op"]
    if op == "train_forward":
        return train.forward(s["x"], s["wg"], s["wu"], s["wd"], workspace=s["workspace"], **_activation(case))
    if op == "train_backward":
        return train.backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], s["g"], s["u"], workspace=s["workspace"],
                              **_activation(case))
    if op == "norm":
        return block_norm.forward(s["y"], s["res"], w_pre=s["w_pre"], w_post=s["w_post"], gate=s["gate"],
                                  post=case["post"], res_scale=case["res_scale"], eps=EPS)
    if op == "norm_backward":
        return block_norm.backward(s["dxn"], s["dr"], s["y"], s["r"], w_pre=s["w_pre"], w_post=s["w_post"],
                                   gate=s["gate"], post=case["post"], res_scale=case["res_scale"], eps=EPS,
                                   workspace=s["workspace"])
    if op == "w4_forward":
        return w4.forward(s["x"], *s["w"], workspace=s["workspace"], **_activation(case))
    return w4.matmul(s["x"], s["w"][0], workspace=s["workspace"])


# ---- the plain forms -------------------------------------------------------------


def _bf16(*tensors):
    return tuple(t if t is None else t.to(torch.bfloat16) for t in tensors)


def _act(g, activation):
    """act(g) and its derivative."""
    beta = BETA if activation == "swish" else 1.0
    s = 1 / (1 + torch.exp(-beta * g))
    if activation == "sigmoid":
        return s, s * (1 - s)
    return g * s, s + beta * g * s * (1 - s)


def _dequantised(q, scale, zero, group):
    rows = torch.arange(q.shape[0], device=q.device) // group
    return (q.float() - zero.float()[rows]) * scale.float()[rows]


def _rms(x):
    return 1 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op = case["op"]
    if op == "train_forward":
        x = s["x"].float()
        g, u = x @ s["wg"].float(), x @ s["wu"].float()
        y = (_act(g, case["activation"])[0] * u) @ s["wd"].float()
        return _bf16(y, g, u)
    if op == "train_backward":
        x, g, u, dy = s["x"].float(), s["g"].float(), s["u"].float(), s["dy"].float()
        a, da = _act(g, case["activation"])
        dh = dy @ s["wd"].float().t()
        dg, du = dh * u * da, dh * a
        dx = dg @ s["wg"].float().t() + du @ s["wu"].float().t()
        return _bf16(dx, x.t() @ dg, x.t() @ du, (a * u).t() @ dy)
    if op == "norm":
        z = s["y"].float()
        if case["post"]:
            z = z * _rms(z) * s["w_post"].float()
        if s["gate"] is not None:
            z = z * s["gate"].float()
        r = case["res_scale"] * s["res"].float() + z
        return r.to(s["res"].dtype), (r * _rms(r) * s["w_pre"].float()).to(torch.bfloat16)
    if op == "norm_backward":
        y, r, dxn = s["y"].float(), s["r"].float(), s["dxn"].float()
        rr = _rms(r)
        xhat, a = r * rr, dxn * s["w_pre"].float()
        total = s["dr"].float() + rr * (a - xhat * (a * xhat).mean(dim=1, keepdim=True))
        dw_pre = (dxn * xhat).double().sum(dim=0)
        dz = total if s["gate"] is None else total * s["gate"].float()
        dw_post, z = None, y
        if case["post"]:
            ry = _rms(y)
            yhat, b = y * ry, dz * s["w_post"].float()
            z = yhat * s["w_post"].float()
            dw_post = (dz * yhat).double().sum(dim=0)
            dy = ry * (b - yhat * (b * yhat).mean(dim=1, keepdim=True))
        else:
            dy = dz
        dgate = None if s["gate"] is None else total * z
        if case["gate"] == "channel":
            dgate = dgate.double().sum(dim=0)
        dres = (case["res_scale"] * total).to(s["r"].dtype)
        dy, dw_pre, dw_post, dgate = _bf16(dy, dw_pre, dw_post, dgate)
        return dy, dres, dw_pre, dw_post, dgate
    w = [_dequantised(*t, case["group"]) for t in s["w"]]
    x = s["x"].float()
    if op == "w4_matmul":
        return (x @ w[0]).to(torch.bfloat16)
    return ((_act(x @ w[0], case["activation"])[0] * (x @ w[1])) @ w[2]).to(torch.bfloat16)


# ---- the definitions in 64 bits ----------------------------------------------------


def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op.startswith("w4"):
        x = t["x"].double()
        w = []
        for q, scale, zero in t["w"]:
            step = scale.double().repeat_interleave(case["group"], dim=0)[:q.shape[0]]
            w.append((q.double() - zero.double().repeat_interleave(case["group"], dim=0)[:q.shape[0]]) * step)
        if op == "w4_matmul":
            return x.matmul(w[0])
        g = x.matmul(w[0])
        h = torch.sigmoid(g * (BETA if case["activation"] == "swish" else 1.0)) * x.matmul(w[1])
        return (h if case["activation"] == "sigmoid" else g * h).matmul(w[2])
    d = {k: v if v is None else v.double() for k, v in t.items()}
    if op.startswith("train"):
        beta = BETA if case["activation"] == "swish" else 1.0
        g = d["x"].matmul(d["wg"]) if op == "train_forward" else d["g"]
        u = d["x"].matmul(d["wu"]) if op == "train_forward" else d["u"]
        s = torch.sigmoid(beta * g)
        gated = s if case["activation"] == "sigmoid" else g * s
        if op == "train_forward":
            return (gated * u).matmul(d["wd"]), g, u
        slope = s * torch.sigmoid(-beta * g)
        if case["activation"] != "sigmoid":
            slope = s + beta * g * slope
        dh = torch.matmul(d["dy"], d["wd"].mT)
        dg, du = dh * u * slope, dh * gated
        dx = torch.matmul(torch.cat([dg, du], dim=1), torch.cat([d["wg"], d["wu"]], dim=1).mT)
        return dx, d["x"].mT.matmul(dg), d["x"].mT.matmul(du), (gated * u).mT.matmul(d["dy"])
    rms = lambda v: torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS)  # noqa: E731
    gate = 1.0 if d["gate"] is None else d["gate"]
    y, D = d["y"], case["D"]
    yn = y * rms(y) if case["post"] else y
    gain = d["w_post"] if case["post"] else 1.0
    if op == "norm":
        r = case["res_scale"] * d["res"] + gate * gain * yn
        return r, r * rms(r) * d["w_pre"]
    # The Jacobian of v / rms(v) applied to c: c / rms - v (v . c) / (D rms^3).
    back = lambda v, c: rms(v) * c - v * rms(v) ** 3 * (v * c).sum(dim=1, keepdim=True) / D  # noqa: E731
    r = d["r"]
    total = d["dr"] + back(r, d["dxn"] * d["w_pre"])
    dyn = total * gate * gain
    dgate = total * yn * gain
    return (back(y, dyn) if case["post"] else dyn, case["res_scale"] * total, (d["dxn"] * r * rms(r)).sum(dim=0),
            (total * gate * yn).sum(dim=0) if case["post"] else None,
            None if case["gate"] == "none" else dgate.sum(dim=0) if case["gate"] == "channel" else dgate)
