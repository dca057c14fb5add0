"""The operators of a block whose MLP is sparse: tokens sorted by expert and
back, the experts' Gated MLPs over the sorted rows, and dropout on the way into
the residual stream.

A case is a dict of plain values; "op" is one of

    dispatch          the sort (offsets, slots) and the sorted rows xs
    combine           y = sum over a token's experts of weight times row; without
                      weights it is the gradient of dispatch
    combine_backward  the gradients of the rows and of the weights
    experts           the Gated MLP of each expert over its rows, with "keep" the
                      forward pass of training, which returns G and U too
    experts_backward  the gradients of the rows and of the three weights
    dropout           out = res + kept x / (1 - p); with "backward" its gradient

`run` computes a case in plain 32-bit torch operations, or with `own` true by
the library's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

BETA = 1.702  # the swish slope of the SwiGLU variant
LARGEST = (4096, 2, 8, 4096, 14336)  # T, k, E, D, F of the largest listed case
ROUTES = ("dispatch", "combine", "combine_backward")


# ---- cases ---------------------------------------------------------------------


def _route(name, op, T, k, E, D, padded=False, weights="fp32"):
    return {"name": name, "op": op, "T": T, "k": k, "E": E, "D": D, "padded": padded, "weights": weights}


def _experts(name, op, T, k, E, D, F, padded=False, activation="silu", keep=False):
    return {"name": name, "op": op, "T": T, "k": k, "E": E, "D": D, "F": F, "padded": padded,
            "activation": activation, "keep": keep}


def _dropout(name, T, D, p, res="none", backward=False):
    return {"name": name, "op": "dropout", "T": T, "D": D, "p": p, "res": res, "backward": backward}


def listed():
    return [
        # One token of a decoding sequence to 2 experts of 8: bound by latency.
        _route("dispatch_1", "dispatch", 1, 2, 8, 4096),
        # A micro-batch or a prefill chunk to 2 of 8.
        _route("dispatch_4096", "dispatch", 4096, 2, 8, 4096),
        # An odd batch of decoding sequences, 8 of 64 experts, an odd width.
        _route("combine_33", "combine", 33, 8, 64, 2056, weights="bf16"),
        # A micro-batch back from 8 of 64 fine-grained experts.
        _route("combine_4096", "combine", 4096, 8, 64, 4096),
        # A short ragged batch, a quarter of it padding, of a wider model.
        _route("combine_backward_300", "combine_backward", 300, 4, 16, 5120, padded=True),
        # The gradients of a micro-batch over fine-grained experts.
        _route("combine_backward_4096", "combine_backward", 4096, 8, 64, 4096),
        # Single-stream decode of the 8B-class layer with 8 experts: bound by the
        # weights of the two experts.
        _experts("experts_1", "experts", 1, 2, 8, 4096, 14336),
        # The forward pass of a training micro-batch on that layer: bound by the
        # matrix cores.
        _experts("experts_4096", "experts", 4096, 2, 8, 4096, 14336, keep=True),
        # A padded batch on fine-grained experts, few rows for each: bound by the
        # weights read and the weight gradients written.
        _experts("experts_backward_300", "experts_backward", 300, 4, 32, 2048, 1024, padded=True, activation="swish"),
        # The backward pass of the micro-batch.
        _experts("experts_backward_4096", "experts_backward", *LARGEST),
        # The smallest call, a toy layer: bound by latency.
        _dropout("dropout_16", 16, 256, 0.1),
        # A micro-batch's block output into an fp32 residual stream.
        _dropout("dropout_4096", 4096, 4096, 0.1, res="fp32"),
    ]


# (D, F) of the repository's workloads and tests, and of the same class; the
# narrow ones are fine-grained experts.
_WIDTHS = [(256, 512), (1024, 512), (1024, 4096), (1032, 2056), (2048, 768), (2048, 1024), (2048, 1408), (2048, 8192),
           (4096, 1536), (4096, 2048), (4096, 14336), (4096, 16384), (5120, 1536), (5120, 13824)]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    most = work(_experts("", "experts_backward", *LARGEST))
    while True:
        op = rng.choice(["dispatch", "combine", "combine_backward", "experts", "experts_backward", "experts",
                         "experts_backward", "dropout"])
        k = rng.choice([1, 2, 2, 4, 6, 8, 8])
        E = rng.choice([8, 8, 16, 32, 60, 64, 128, 256])
        if op in ROUTES:
            weights = "none" if op == "combine" and rng.random() < 0.3 else rng.choice(["fp32", "fp32", "bf16"])
            c = _route("", op, _log_uniform(rng, 1, 8192), k, E, 8 * _log_uniform(rng, 32, 1024), rng.random() < 0.3,
                       weights)
        elif op == "dropout":
            backward = rng.random() < 0.4
            res = rng.choice(["bf16", "fp32"]) if backward else rng.choice(["none", "bf16", "fp32"])
            c = _dropout("", _log_uniform(rng, 1, 8192), 8 * _log_uniform(rng, 32, 1024),
                         rng.choice([0.05, 0.1, 0.1, 0.3, 0.5]), res, backward)
        else:
            D, F = rng.choice(_WIDTHS)
            if rng.random() < 0.3:  # widths of no particular class
                D = 8 * _log_uniform(rng, 32, 512)
                F = 8 * _log_uniform(rng, 32, 1024)
            c = _experts("", op, _log_uniform(rng, 1, 4096), k, E, D, F, rng.random() < 0.3,
                         rng.choice(["silu", "silu", "swish", "sigmoid"]), op == "experts" and rng.random() < 0.5)
        del c["name"]
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and \
                c.get("E", 1) * c["D"] * c.get("F", 1) <= LARGEST[2] * LARGEST[3] * LARGEST[4]:
            return c


def _tokens(case):
    """Tokens with experts: of a padded batch, the last quarter has none."""
    return case["T"] - case["T"] // 4 if case["padded"] else case["T"]


def work(case):
    op, T, D = case["op"], case["T"], case["D"]
    if op == "dropout":
        # x in, out out; a residual stream in, or the gradient of one in fp32.
        b = {"none": 2, "bf16": 2, "fp32": 4}[case["res"]]
        per = b + 2 if case["backward"] else 2 + b + (b if case["res"] != "none" else 0)
        return {"bytes": float(per * T * D), "flops": 20.0 * T * D}
    k, E = case["k"], case["E"]
    rows, N = _tokens(case) * k, T * k
    wb = {"fp32": 4, "bf16": 2, "none": 0}[case.get("weights", "none")]
    if op == "dispatch":
        return {"bytes": 2.0 * D * (_tokens(case) + rows) + 12.0 * N + 4 * (E + 1), "flops": 4.0 * N}
    if op == "combine":
        return {"bytes": 2.0 * D * (T + rows) + (4.0 + wb) * N, "flops": 2.0 * rows * D}
    if op == "combine_backward":
        return {"bytes": 2.0 * D * (_tokens(case) + 2 * rows) + (4.0 + 2 * wb) * N, "flops": 3.0 * rows * D}
    F = case["F"]
    # Experts that some token is expected to go to.
    active = E * (1.0 - (1.0 - k / E) ** _tokens(case))
    if op == "experts":
        return {"bytes": 6.0 * active * D * F + 4.0 * rows * D + (4.0 * rows * F if case["keep"] else 0.0),
                "flops": 6.0 * rows * D * F}
    return {"bytes": 6.0 * (active + E) * D * F + 6.0 * rows * D + 4.0 * rows * F, "flops": 12.0 * rows * D * F}


# ---- inputs --------------------------------------------------------------------


def _normal(gen, rows, cols, scale=1.0, dtype=torch.bfloat16):
    t = torch.empty((rows, cols), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // cols)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        t[r:r + n] = torch.randn((n, cols), generator=gen, device="cuda") * scale
    return t


def _routing(gen, case):
    """ids [T, k] int64 of the k likeliest experts of a router with a preference
    for some of them, -1 in padding, and their weights [T, k], which add up to 1."""
    T, k, E = case["T"], case["k"], case["E"]
    logits = torch.randn((T, E), generator=gen, device="cuda") + 0.5 * torch.randn(E, generator=gen, device="cuda")
    top = logits.sort(dim=1, descending=True)
    ids, w = top.indices[:, :k].contiguous(), top.values[:, :k].exp()
    w = w / w.sum(dim=1, keepdim=True)
    ids[_tokens(case):] = -1
    return ids, w.to(torch.bfloat16 if case.get("weights") == "bf16" else torch.float32)


def _sorted(ids, E):
    """(offsets [E + 1], slots [T, k]) int32: where each expert's rows begin, and the
    row of every assignment, in the order of the assignments within an expert; -1 for
    one without an expert."""
    flat = ids.reshape(-1)
    hit = torch.arange(E, device=ids.device)[:, None] == flat
    count = hit.long().cumsum(dim=1)
    offsets = torch.zeros(E + 1, dtype=torch.long, device=ids.device)
    offsets[1:] = count[:, -1].cumsum(dim=0)
    valid = (flat >= 0) & (flat < E)
    e = torch.where(valid, flat, 0)
    slots = offsets[e] + count.gather(0, e[None])[0] - 1
    return offsets.int(), torch.where(valid, slots, -1).int().view(ids.shape)


def _inputs(case, seed):
    """Activations and gradients N(0, 1), weights N(0, 1/fan_in); G and U, products
    of such, N(0, 1) as well.  Rows behind the last expert's are zeros."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, T, D = case["op"], case["T"], case["D"]
    if op == "dropout":
        res = torch.float32 if case["res"] == "fp32" else torch.bfloat16
        t = {"seed": int(np.random.default_rng(seed).integers(1 << 62)), "offset": 5 + (seed % 1000) * (1 << 30)}
        if case["backward"]:
            t["dout"] = _normal(gen, T, D, dtype=res)
        else:
            t["x"] = _normal(gen, T, D)
            t["res"] = None if case["res"] == "none" else _normal(gen, T, D, 2.0, dtype=res)
        return t
    E, N = case["E"], T * case["k"]
    ids, weights = _routing(gen, case)
    t = {"ids": ids}
    t["offsets"], t["slots"] = _sorted(ids, E)
    if op == "dispatch":
        t["x"] = _normal(gen, T, D)
        return t
    rows = _tokens(case) * case["k"]

    def sorted_rows(cols):
        r = _normal(gen, N, cols)
        r[rows:] = 0
        return r

    if op in ROUTES:
        t["weights"] = None if case["weights"] == "none" else weights
        t["ys"] = sorted_rows(D)
        if op == "combine_backward":
            t["dy"] = _normal(gen, T, D)
        return t
    F = case["F"]
    t["xs"] = sorted_rows(D)
    t["wg"] = _normal(gen, E * D, F, D ** -0.5).view(E, D, F)
    t["wu"] = _normal(gen, E * D, F, D ** -0.5).view(E, D, F)
    t["wd"] = _normal(gen, E * F, D, F ** -0.5).view(E, F, D)
    if op == "experts_backward":
        t.update(g=sorted_rows(F), u=sorted_rows(F), dys=sorted_rows(D))
    return t


def _activation(case):
    kw = {"activation": case["activation"]}
    if case["activation"] == "swish":
        kw["beta"] = BETA
    return kw


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "dropout":
        return s
    T, D, N = case["T"], case["D"], case["T"] * case["k"]
    zeros = lambda rows, cols: torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    # Buffers of sorted rows, as a program keeps them: those behind the last expert's
    # rows are not written.
    if op in ("dispatch", "combine_backward", "experts", "experts_backward"):
        s["out"] = zeros(N, D)
    if op == "experts" and case["keep"]:
        s["g"], s["u"] = zeros(N, case["F"]), zeros(N, case["F"])
    if own:
        if op.startswith("experts"):
            from paper_2606_26344_amd import experts

            s["workspace"] = experts.make_workspace(N, case["E"], D, case["F"])
    elif op.startswith("experts"):
        s["bounds"] = s["offsets"].tolist()  # the plain form's loop over experts
    return s


# ---- the library's calls ---------------------------------------------------------


def _run_own(s):
    from paper_2606_26344_amd import dropout, experts, route

    case = s["case"]
    op = case["op"]
    if op == "dispatch":
        offsets, slots = route.sort(s["ids"], case["E"])
        return offsets, slots, route.dispatch(s["x"], slots, out=s["out"])
    if op == "combine":
        return route.combine(s["ys"], s["slots"], s["weights"])
    if op == "combine_backward":
        return route.combine_backward(s["dy"], s["ys"], s["slots"], s["weights"], dys=s["out"])
    if op == "dropout":
        if case["backward"]:
            return dropout.backward(s["dout"], case["p"], s["seed"], offset=s["offset"])
        return dropout.forward(s["x"], case["p"], s["seed"], offset=s["offset"], res=s["res"])
    w = (s["wg"], s["wu"], s["wd"])
    kw = dict(workspace=s["workspace"], **_activation(case))
    if op == "experts_backward":
        return experts.backward(s["dys"], s["xs"], s["offsets"], *w, s["g"], s["u"], dxs=s["out"], **kw)
    if case["keep"]:
        return experts.train_forward(s["xs"], s["offsets"], *w, out=s["out"], g=s["g"], u=s["u"], **kw)
    return experts.forward(s["xs"], s["offsets"], *w, out=s["out"], **kw)


# ---- the plain forms -------------------------------------------------------------


def _act(g, activation):
    """act(g) and its derivative."""
    beta = BETA if activation == "swish" else 1.0
    s = 1 / (1 + torch.exp(-beta * g))
    if activation == "sigmoid":
        return s, s * (1 - s)
    return g * s, s + beta * g * s * (1 - s)


def _kept(groups, seed, offset, p, device):
    """Which elements of groups of eight are kept, and the factor 1 / (1 - p): 16 bits
    for each of Philox4x32-10 (Salmon et al., 2011) with the group's number as counter."""
    mask = 0xffffffff
    c = torch.arange(groups, dtype=torch.long, device=device) + offset
    x = [c & mask, (c >> 32) & mask, torch.zeros_like(c), torch.zeros_like(c)]
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        # 32 x 32 bit products, whose low 64 bits wrap as they should.
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [((b >> 32) & mask) ^ x[1] ^ k0, b & mask, ((a >> 32) & mask) ^ x[3] ^ k1, a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    bits = torch.stack([h for w in x for h in (w & 0xffff, w >> 16)], dim=1)
    threshold = round(p * 65536)
    return bits >= threshold, 65536 / (65536 - threshold)


def _taken(rows, slots):
    """rows[slots] in 32 bits, zeros where there is no slot."""
    got = rows[slots.clamp(min=0).long()].float()
    return torch.where((slots >= 0)[..., None], got, 0.0)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op = case["op"]
    if op == "dispatch":
        offsets, slots = _sorted(s["ids"], case["E"])
        # One row more takes what has no slot.
        xs = torch.zeros((slots.numel() + 1, case["D"]), dtype=s["x"].dtype, device="cuda")
        xs[torch.where(slots < 0, slots.numel(), slots).long()] = s["x"][:, None]
        return offsets, slots, xs[:-1]
    if op == "combine":
        y = torch.zeros((case["T"], case["D"]), device="cuda")
        for j in range(case["k"]):
            rows = _taken(s["ys"], s["slots"][:, j])
            y = y + (rows if s["weights"] is None else rows * s["weights"][:, j, None].float())
        return y.to(torch.bfloat16)
    if op == "combine_backward":
        dy = s["dy"].float()
        dys = torch.zeros((s["slots"].numel() + 1, case["D"]), dtype=torch.bfloat16, device="cuda")
        dw = []
        for j in range(case["k"]):
            slot = s["slots"][:, j]
            at = torch.where(slot < 0, s["slots"].numel(), slot).long()
            dys[at] = (dy * s["weights"][:, j, None].float()).to(torch.bfloat16)
            dw.append((dy * _taken(s["ys"], slot)).sum(dim=1))
        dys[-1] = 0
        return dys[:-1], torch.stack(dw, dim=1).to(s["weights"].dtype)
    if op == "dropout":
        x = (s["dout"] if case["backward"] else s["x"])
        kept, factor = _kept(x.numel() // 8, s["seed"], s["offset"], case["p"], x.device)
        out = torch.where(kept.view(x.shape), x.float() * factor, 0.0)
        if case["backward"] or s["res"] is None:
            return out.to(torch.bfloat16)
        return (s["res"].float() + out).to(s["res"].dtype)
    bf16 = torch.bfloat16
    bounds = s["bounds"]
    if op == "experts":
        out = s["out"]
        for e in range(case["E"]):
            part = slice(bounds[e], bounds[e + 1])
            if part.start == part.stop:
                continue
            x = s["xs"][part].float()
            g, u = x @ s["wg"][e].float(), x @ s["wu"][e].float()
            out[part] = ((_act(g, case["activation"])[0] * u) @ s["wd"][e].float()).to(bf16)
            if case["keep"]:
                s["g"][part], s["u"][part] = g.to(bf16), u.to(bf16)
        return (out, s["g"], s["u"]) if case["keep"] else out
    dxs = s["out"]
    dw = [torch.zeros_like(s[n]) for n in ("wg", "wu", "wd")]
    for e in range(case["E"]):
        part = slice(bounds[e], bounds[e + 1])
        if part.start == part.stop:
            continue
        x, g, u, dy = (s[n][part].float() for n in ("xs", "g", "u", "dys"))
        a, da = _act(g, case["activation"])
        dh = dy @ s["wd"][e].float().t()
        dg, du = dh * u * da, dh * a
        dxs[part] = (dg @ s["wg"][e].float().t() + du @ s["wu"][e].float().t()).to(bf16)
        dw[0][e], dw[1][e], dw[2][e] = (x.t() @ dg).to(bf16), (x.t() @ du).to(bf16), ((a * u).t() @ dy).to(bf16)
    return (dxs, *dw)


# ---- the definitions in 64 bits ----------------------------------------------------


def _exact_sort(ids, E):
    """As _sorted, by a stable sort on the host."""
    flat = ids.cpu().numpy().reshape(-1)
    key = np.where((flat < 0) | (flat >= E), E, flat)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(E + 1), side="left").astype(np.int32)
    slots = np.empty(flat.size, dtype=np.int32)
    slots[order] = np.arange(flat.size, dtype=np.int32)
    slots[key == E] = -1
    return offsets, slots


def _exact_bits(groups, seed, offset):
    """16 bits of every element, in 64-bit unsigned integers on the host."""
    u = np.uint64
    low, half = u(0xffffffff), u(32)
    n = np.arange(groups, dtype=np.uint64) + u(offset)
    ctr = np.stack([n & low, n >> half, np.zeros_like(n), np.zeros_like(n)])
    key = [seed & 0xffffffff, seed >> 32]
    for r in range(10):
        ka, kb = u((key[0] + r * 0x9E3779B9) % 2 ** 32), u((key[1] + r * 0xBB67AE85) % 2 ** 32)
        first, second = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = np.stack([second >> half ^ ctr[1] ^ ka, second & low, first >> half ^ ctr[3] ^ kb, first & low])
    return ctr.astype(np.uint32).T.copy().view(np.uint16)  # the low half of a word first


def exact(case, seed):
    t = _inputs(case, seed)
    op = case["op"]
    if op == "dropout":
        v = t["dout"] if case["backward"] else t["x"]
        cut = round(case["p"] * 65536)
        kept = torch.from_numpy((_exact_bits(v.numel() // 8, t["seed"], t["offset"]) >= cut).reshape(v.shape)).cuda()
        out = v.double() / (1.0 - cut / 65536) * kept
        return out if case["backward"] or t["res"] is None else out + t["res"].double()
    if op == "dispatch":
        offsets, slots = _exact_sort(t["ids"], case["E"])
        xs = torch.zeros((slots.size, case["D"]), dtype=torch.float64, device="cuda")
        some = np.flatnonzero(slots >= 0)
        token = torch.from_numpy(some // case["k"]).cuda()
        xs[torch.from_numpy(slots[some]).long().cuda()] = t["x"].double()[token]
        return (torch.from_numpy(offsets).cuda(), torch.from_numpy(slots).view(t["ids"].shape).cuda(), xs)
    if op in ROUTES:
        live = _tokens(case)
        at = t["slots"][:live].long()
        w = torch.ones(at.shape, dtype=torch.float64, device="cuda") if t["weights"] is None else t["weights"][:live].double()
        if op == "combine":
            y = torch.zeros((case["T"], case["D"]), dtype=torch.float64, device="cuda")
            for j in range(case["k"]):
                y[:live].addcmul_(t["ys"][at[:, j]].double(), w[:, j:j + 1])
            return y
        dys = torch.zeros(t["ys"].shape, dtype=torch.float64, device="cuda")
        dw = torch.zeros(t["slots"].shape, dtype=torch.float64, device="cuda")
        dy = t["dy"][:live].double()
        for j in range(case["k"]):
            dys.index_copy_(0, at[:, j], dy * w[:, j:j + 1])
            dw[:live, j] = torch.linalg.vecdot(dy, t["ys"][at[:, j]].double())
        return dys, dw
    beta = BETA if case["activation"] == "swish" else 1.0
    ends = t["offsets"].tolist()
    N, D, F = t["xs"].shape[0], case["D"], case["F"]
    rows = lambda cols: torch.zeros((N, cols), dtype=torch.float64, device="cuda")  # noqa: E731
    if op == "experts":
        y, kept = rows(D), [rows(F), rows(F)] if case["keep"] else None
        for e in range(case["E"]):
            lo, hi = ends[e], ends[e + 1]
            if hi > lo:
                x = t["xs"][lo:hi].double()
                g, u = x.matmul(t["wg"][e].double()), x.matmul(t["wu"][e].double())
                h = torch.sigmoid(beta * g) * u
                y[lo:hi] = (h if case["activation"] == "sigmoid" else g * h).matmul(t["wd"][e].double())
                if kept:
                    kept[0][lo:hi], kept[1][lo:hi] = g, u
        return (y, *kept) if kept else y
    dx = rows(D)
    dwg, dwu, dwd = (torch.zeros(t[n].shape, dtype=torch.float64, device="cuda") for n in ("wg", "wu", "wd"))
    for e in range(case["E"]):
        lo, hi = ends[e], ends[e + 1]
        if hi == lo:
            continue
        x, g, u, dy = (t[n][lo:hi].double() for n in ("xs", "g", "u", "dys"))
        s = torch.sigmoid(beta * g)
        gated = s if case["activation"] == "sigmoid" else g * s
        slope = s * torch.sigmoid(-beta * g)
        if case["activation"] != "sigmoid":
            slope = s + beta * g * slope
        dh = dy.matmul(t["wd"][e].double().mT.contiguous())
        dg, du = dh * u * slope, dh * gated
        dx[lo:hi] = torch.matmul(dg, t["wg"][e].double().mT) + torch.matmul(du, t["wu"][e].double().mT)
        dwg[e], dwu[e], dwd[e] = x.mT.matmul(dg), x.mT.matmul(du), (gated * u).mT.matmul(dy)
    return dx, dwg, dwu, dwd
