"""Performance cases of the dense operators beside the MACE step.

A program that trains or serves a species-routed head next to the library's
energies (a readout on expert layers, a small network distilled from a MACE
teacher, a fine-tuned linear) calls three operators:

* `linear`: y = act(x W_g + b_g) + r, one weight block per group of rows, and
  its backward pass;
* `route`: the stable sort of (row, slot) pairs by expert, the rows gathered in
  that order and combined again with weights, and the gradients of both;
* `orthogonalise`: the Newton-Schulz iteration x <- a x + (b A + c A^2) x,
  A = x x^T, over a batch of weight gradients.

The plain forms below are elementary torch operations in FP32, rounded once
per output; `exact` is written from the definitions in FP64.  Sizes are the
library's own (K = 32 to 128 channels, a 64-wide radial network with P K
outputs, water boxes of 96 to 36,864 atoms, up to ten species) and, beside
them, generic widths up to 2048 and up to 64 experts.
"""
from __future__ import annotations

import math

import torch

own = False   # True: the library's kernels; False: the plain forms

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5   # a, b, c of five Newton-Schulz steps
EPS = 1e-7
MAX_LINEAR_FLOPS = 6.0 * 36864 * 2048 * 2048
MAX_ROUTE_ELEMENTS = 36864 * 8 * 1024
MAX_ORTHOGONALISE_FLOPS = 2 * 30.0 * 2048 ** 3


def _linear(rows, n_in, n_out, groups, dtype, act, train, bias=True, residual=False):
    return {"op": "linear", "rows": rows, "n_in": n_in, "n_out": n_out, "groups": groups, "dtype": dtype, "act": act,
            "train": train, "bias": bias, "residual": residual}


def _route(tokens, top_k, experts, width, dtype, train, dropped=False):
    return {"op": "route", "tokens": tokens, "top_k": top_k, "experts": experts, "width": width, "dtype": dtype,
            "train": train, "dropped": dropped}


def _orthogonalise(batch, rows, cols, dtype):
    return {"op": "orthogonalise", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # the residual head on one atom: a single call's latency
        dict(_linear(1, 128, 128, 1, "fp32", "silu", False, residual=True), name="linear_row1_128_fp32"),
        # the radial network's last layer over the edges of a 1,536-atom box, FP32, no bias
        dict(_linear(81920, 64, 1280, 1, "fp32", "none", False, bias=False), name="linear_81920_64x1280_fp32"),
        # a training step of a species-routed layer on ragged sizes that no tile divides, ten species
        dict(_linear(17711, 97, 211, 10, "fp16", "gelu", True), name="linear_train_17711_97x211_fp16"),
        # a training step of a wide hidden layer on the atoms of the large box, eight experts
        dict(_linear(36864, 2048, 2048, 8, "bf16", "silu", True, residual=True), name="linear_train_36864_2048_bf16"),
        # a small box routed by its two species: serving, all latency
        dict(_route(96, 1, 2, 128, "fp32", False), name="route_96_top1_fp32"),
        # a medium box, two experts of sixteen each, forward and backward
        dict(_route(4608, 2, 16, 512, "bf16", True), name="route_train_4608_top2_bf16"),
        # odd width and expert count, a tenth of the slots dropped
        dict(_route(5003, 3, 37, 515, "fp32", True, dropped=True), name="route_train_5003_top3_fp32"),
        # the large box, eight experts of 64 each: memory
        dict(_route(36864, 8, 64, 1024, "bf16", True), name="route_train_36864_top8_bf16"),
        # one 64 x 64 radial layer
        dict(_orthogonalise(1, 64, 64, "fp32"), name="orthogonalise_1x64x64_fp32"),
        # every K x K block of the two-layer l <= 1 model at once
        dict(_orthogonalise(30, 128, 128, "fp32"), name="orthogonalise_30x128x128_fp32"),
        # odd, tall blocks, one per species
        dict(_orthogonalise(10, 515, 211, "bf16"), name="orthogonalise_10x515x211_bf16"),
        # two wide square layers: matrix products alone
        dict(_orthogonalise(2, 2048, 2048, "bf16"), name="orthogonalise_2x2048x2048_bf16"),
    ]


def _log_int(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5))))))


def draw(rng):
    op = rng.choice(["linear", "route", "orthogonalise"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    while True:
        if op == "linear":
            c = _linear(_log_int(rng, 1, 131072), _log_int(rng, 16, 2048), _log_int(rng, 16, 2048),
                        _log_int(rng, 1, 16), dtype, rng.choice(["none", "silu", "gelu"]), rng.random() < 0.5,
                        rng.random() < 0.7, rng.random() < 0.5)
            if work(c)["flops"] <= MAX_LINEAR_FLOPS:
                return c
        elif op == "route":
            k = rng.randint(1, 8)
            c = _route(_log_int(rng, 1, 65536), k, _log_int(rng, max(2, k), 256), _log_int(rng, 16, 2048), dtype,
                       rng.random() < 0.6, rng.random() < 0.3)
            if c["tokens"] * k * c["width"] * SIZE[dtype] <= MAX_ROUTE_ELEMENTS * 2:
                return c
        else:
            c = _orthogonalise(_log_int(rng, 1, 128), _log_int(rng, 8, 2048), _log_int(rng, 8, 2048), dtype)
            if work(c)["flops"] <= MAX_ORTHOGONALISE_FLOPS:
                return c


def work(case):
    b = SIZE[case["dtype"]]
    if case["op"] == "linear":
        n, ki, ko, g = case["rows"], case["n_in"], case["n_out"], case["groups"]
        used = min(g, n) * (ki * ko + (ko if case["bias"] else 0))   # weights of groups that have rows
        size = n * ki + used + n * ko * (2 if case["residual"] else 1)
        flops = 2.0 * n * ki * ko
        if case["train"]:   # dy read; dx, dW and db written
            size += n * ko + n * ki + g * (ki * ko + (ko if case["bias"] else 0))
            flops *= 3.0
        return {"bytes": float(size * b), "flops": flops}
    if case["op"] == "route":
        n, k, d = case["tokens"], case["top_k"], case["width"]
        index = 4.0 * (3 * n * k + case["experts"] + 1) + 4.0 * n * k   # experts in, both orders out; weights
        size = 2.0 * n * d + 2.0 * n * k * d   # x, out; gathered rows, rows to combine
        flops = 2.0 * n * k * d
        if case["train"]:   # dout, dx; the gradient rows out and in; rows to combine are shared with the forward
            size += 2.0 * n * d + 2.0 * n * k * d
            index += 4.0 * n * k
            flops += 4.0 * n * k * d
        return {"bytes": size * b + index, "flops": flops}
    n, m, w = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # x x^T and A A are symmetric: half of each
    return {"bytes": 2.0 * n * m * w * b, "flops": len(COEFFICIENTS) * n * (3.0 * m * m * w + 1.0 * m ** 3)}


def _groups(n, groups, gen):
    """Row offsets of `groups` contiguous groups of uneven size, and the largest one's size."""
    share = torch.rand(groups, generator=gen) + 0.5
    cut = torch.floor(torch.cumsum(share, 0) / share.sum() * n).to(torch.int64)
    cut[-1] = n
    off = torch.cat([torch.zeros(1, dtype=torch.int64), cut])
    return off.to(torch.int32), int((off[1:] - off[:-1]).max())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dt)

    s = dict(case)
    if case["op"] == "linear":
        n, ki, ko, g = case["rows"], case["n_in"], case["n_out"], case["groups"]
        s["x"] = normal(n, ki)
        s["w"] = normal(g, ki, ko, scale=ki ** -0.5)   # the library's initialisation, N(0, 1) / sqrt(fan in)
        s["b"] = normal(g, ko, scale=0.3) if case["bias"] else None
        s["r"] = normal(n, ko) if case["residual"] else None
        s["offsets"], s["largest"] = None, n
        if g > 1:
            off, s["largest"] = _groups(n, g, host)
            s["offsets"] = off.cuda()
        if case["train"]:
            s["dy"] = normal(n, ko, scale=0.1)
    elif case["op"] == "route":
        n, k, e, d = case["tokens"], case["top_k"], case["experts"], case["width"]
        score = torch.randn(n, e, generator=gen, device="cuda") + torch.linspace(0, 1.5, e, device="cuda")
        top, index = torch.topk(score, k, dim=1)   # distinct experts per row, some far more wanted than others
        s["expert"] = index.to(torch.int32)
        if case["dropped"]:
            gone = torch.rand(n, k, generator=gen, device="cuda") < 0.1
            s["expert"] = torch.where(gone, torch.full_like(s["expert"], -1), s["expert"])
        s["weights"] = torch.softmax(top, dim=1)
        s["x"], s["y_rows"] = normal(n, d), normal(n * k, d)
        if case["train"]:
            s["dout"], s["dx_rows"] = normal(n, d, scale=0.1), normal(n * k, d, scale=0.1)
    else:
        b, m, w = case["batch"], case["rows"], case["cols"]
        r = max(1, min(m, w) // 4)   # a gradient: a few strong directions above noise
        u, v = torch.randn(b, m, r, generator=gen, device="cuda"), torch.randn(b, r, w, generator=gen, device="cuda")
        g = torch.bmm(u, v) * r ** -0.5 + 0.2 * torch.randn(b, m, w, generator=gen, device="cuda")
        s["g"] = (g * 0.01).to(dt)
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"linear": _plain_linear, "route": _plain_route, "orthogonalise": _plain_orthogonalise}[s["op"]](s)


def _run_own(s):
    from paper_2510_23621_amd import layers
    if s["op"] == "linear":
        if not s["train"]:
            return {"y": layers.linear(s["x"], s["w"], s["b"], s["r"], offsets=s["offsets"], act=s["act"])}
        y, z = layers.linear(s["x"], s["w"], s["b"], s["r"], offsets=s["offsets"], act=s["act"], save=True)
        dx, dw, db = layers.linear_backward(s["dy"], s["x"], s["w"], z, offsets=s["offsets"], act=s["act"],
                                            bias=s["bias"])
        return {"y": y, "dx": dx, "dw": dw} | ({"db": db} if s["bias"] else {})
    if s["op"] == "route":
        plan = layers.route(s["expert"], s["experts"])
        out = {"slot_of_row": plan.slot_of_row, "row_of_slot": plan.row_of_slot, "offsets": plan.offsets,
               "rows": layers.route_rows(s["x"], plan), "out": layers.combine_rows(s["y_rows"], plan, s["weights"])}
        if s["train"]:
            out["drows"], out["dweights"] = layers.combine_rows_backward(s["dout"], s["y_rows"], plan, s["weights"])
            out["dx"] = layers.route_rows_backward(s["dx_rows"], plan)
        return out
    return {"y": layers.orthogonalise(s["g"], COEFFICIENTS, eps=EPS)}


# ------------------------------------------------------------------ plain forms

def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _act_slope(z, act):
    if act == "silu":
        t = torch.sigmoid(z)
        return t * (1 + z * (1 - t))
    return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5


def _plain_linear(s):
    n, ki, ko, g, cap = s["rows"], s["n_in"], s["n_out"], s["groups"], s["largest"]
    x, w, dt = s["x"].float(), s["w"].float(), s["x"].dtype
    b = s["b"].float() if s["bias"] else None
    if g == 1:
        group = slot = None
        z = x @ w[0]
        if b is not None:
            z = z + b
    else:   # one batched product over the groups, each padded to the largest
        row = torch.arange(n, device=x.device)
        group = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
        slot = group * cap + row - s["offsets"].long()[group]
        xp = x.new_zeros(g * cap, ki)
        xp[slot] = x
        xp = xp.view(g, cap, ki)
        zp = torch.bmm(xp, w)
        if b is not None:
            zp = zp + b[:, None]
        z = zp.view(g * cap, ko)[slot]
    y = _act(z, s["act"])
    if s["residual"]:
        y = y + s["r"].float()
    out = {"y": y.to(dt)}
    if not s["train"]:
        return out
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(z, s["act"])
    if g == 1:
        out["dx"], out["dw"] = (dz @ w[0].t()).to(dt), (x.t() @ dz).to(dt)[None]
        db = dz.sum(0, keepdim=True)
    else:
        dzp = x.new_zeros(g * cap, ko)
        dzp[slot] = dz
        dzp = dzp.view(g, cap, ko)
        out["dx"] = torch.bmm(dzp, w.transpose(1, 2).contiguous()).view(g * cap, ki)[slot].to(dt)
        out["dw"] = torch.bmm(xp.transpose(1, 2).contiguous(), dzp).to(dt)
        db = dzp.sum(1)
    if s["bias"]:
        out["db"] = db.to(dt)
    return out


def _plain_route(s):
    n, k, e, d = s["tokens"], s["top_k"], s["experts"], s["width"]
    dt = s["x"].dtype
    key = s["expert"].reshape(-1).long()
    key = torch.where(key < 0, torch.full_like(key, e), key)   # dropped slots go past the end
    slot_of_row = torch.sort(key, stable=True).indices
    row_of_slot = torch.empty_like(slot_of_row)
    row_of_slot[slot_of_row] = torch.arange(n * k, device=key.device)
    offsets = torch.searchsorted(key[slot_of_row], torch.arange(e + 1, device=key.device))
    kept = (key[slot_of_row] < e).float()[:, None]
    used = (key < e).float().view(n, k)
    weights = s["weights"] * used
    out = {"slot_of_row": slot_of_row.int(), "row_of_slot": row_of_slot.int().view(n, k), "offsets": offsets.int(),
           "rows": (s["x"].float()[slot_of_row // k] * kept).to(dt)}
    y = s["y_rows"].float()[row_of_slot].view(n, k, d)
    out["out"] = (y * weights[..., None]).sum(1).to(dt)
    if s["train"]:
        dout = s["dout"].float()
        out["drows"] = (dout[slot_of_row // k] * weights.view(-1)[slot_of_row][:, None]).to(dt)
        out["dweights"] = (y * dout[:, None]).sum(2) * used
        out["dx"] = (s["dx_rows"].float()[row_of_slot].view(n, k, d) * used[..., None]).sum(1).to(dt)
    return out


def _plain_orthogonalise(s):
    x = s["g"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + EPS)
    for a, b, c in COEFFICIENTS:
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return {"y": (x.transpose(1, 2).contiguous() if tall else x).to(s["g"].dtype)}


# ------------------------------------------------------------------ FP64 definitions

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "route": _exact_route, "orthogonalise": _exact_orthogonalise}[case["op"]](s)


def _exact_linear(s):
    n, g = s["rows"], s["groups"]
    off = [0, n] if g == 1 else s["offsets"].tolist()
    parts = {"y": [], "dx": [], "dw": [], "db": []}
    for e in range(g):
        at = slice(off[e], off[e + 1])
        x, w = s["x"][at].double(), s["w"][e].double()
        z = x @ w
        if s["bias"]:
            z = z + s["b"][e].double()
        if s["act"] == "silu":   # f = z / (1 + exp(-z)), f' = f / z + f (1 - f / z)
            gate = 1 / (1 + torch.exp(-z))
            f, slope = z * gate, gate + z * gate * (1 - gate)
        elif s["act"] == "gelu":   # f = z Phi(z), f' = Phi(z) + z phi(z)
            phi = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
            gate = 0.5 * torch.erfc(-z / math.sqrt(2))
            f, slope = z * gate, gate + z * phi
        else:
            f, slope = z, torch.ones_like(z)
        parts["y"].append(f + s["r"][at].double() if s["residual"] else f)
        if s["train"]:
            dz = s["dy"][at].double() * slope
            parts["dx"].append(dz @ w.t())
            parts["dw"].append(x.t() @ dz)
            parts["db"].append(dz.sum(0))
    out = {"y": torch.cat(parts["y"])}
    if s["train"]:
        out["dx"], out["dw"] = torch.cat(parts["dx"]), torch.stack(parts["dw"])
        if s["bias"]:
            out["db"] = torch.stack(parts["db"])
    return out


def _exact_route(s):
    n, k, e = s["tokens"], s["top_k"], s["experts"]
    key = s["expert"].reshape(-1).cpu()
    lists = [torch.nonzero(key == i).reshape(-1) for i in range(e)] + [torch.nonzero(key < 0).reshape(-1)]
    slots = torch.cat(lists)   # in order of expert, then of slot; the dropped ones last
    count = torch.tensor([0] + [len(p) for p in lists[:-1]])
    offsets = torch.cumsum(count, 0)
    live = int(offsets[-1])
    row = torch.empty_like(slots)
    row[slots] = torch.arange(n * k)
    out = {"slot_of_row": slots.int().cuda(), "row_of_slot": row.int().view(n, k).cuda(), "offsets": offsets.int().cuda()}
    slots, row = slots.cuda(), row.view(n, k).cuda()
    rows = s["x"].double()[slots // k]
    rows[live:] = 0
    out["rows"] = rows
    total = torch.zeros(n, s["width"], dtype=torch.float64, device="cuda")
    for j in range(k):
        on = row[:, j] < live
        total[on] += s["weights"][on, j, None].double() * s["y_rows"][row[on, j]].double()
    out["out"] = total
    if s["train"]:
        drows = torch.zeros(n * k, s["width"], dtype=torch.float64, device="cuda")
        dweights = torch.zeros(n, k, dtype=torch.float64, device="cuda")
        dx = torch.zeros_like(total)
        for j in range(k):
            on = row[:, j] < live
            to, dout = row[on, j], s["dout"][on].double()
            drows[to] = s["weights"][on, j, None].double() * dout
            dweights[on, j] = (s["y_rows"][to].double() * dout).sum(1)
            dx[on] += s["dx_rows"][to].double()
        out["drows"], out["dweights"], out["dx"] = drows, dweights, dx
    return out


def _exact_orthogonalise(s):
    done = []
    for g in s["g"]:   # one matrix at a time; for a tall one the products on the other side, which are the same map
        x = g.double()
        x = x / (torch.linalg.vector_norm(x) + EPS)
        for a, b, c in COEFFICIENTS:
            if x.shape[0] <= x.shape[1]:
                gram = x @ x.t()
                x = a * x + b * (gram @ x) + c * (gram @ (gram @ x))
            else:
                gram = x.t() @ x
                x = a * x + b * (x @ gram) + c * ((x @ gram) @ gram)
        done.append(x)
    return {"y": torch.stack(done)}
