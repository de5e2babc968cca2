"""Distils a MACE teacher's per-atom energies into a small routed network.

The teacher is the library's own model on periodic water; the student sees
radial sums over an atom's neighbours and runs on the dense operators: a
trunk layer, a router that sends each atom to two of four experts, the experts'
two layers as grouped linears, and a linear readout.  Every gradient is one of
the library's backward calls (the router's softmax is differentiated here), and
the weight matrices are updated with orthogonalised momenta.

    python examples/distil_head.py [steps]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_2510_23621_amd import MaceGraph, binding as B, layers as L  # noqa: E402
from synth.configs import make_system, model_params  # noqa: E402

EXPERTS, TOP_K, WIDTH, HIDDEN, RADIAL = 4, 2, 64, 96, 16
MATRICES = ("trunk.w", "router.w", "up.w", "down.w", "read.w")


def teacher_data(boxes=8, jitter=0.03):
    """Descriptors [atoms, 2 RADIAL + 2] and standardised teacher energies [atoms, 1] of jittered water boxes."""
    params = model_params(0)
    desc = B.make_desc(**params)
    lay, _ = B.mace_weight_layout(desc)
    blob = synth.weight_blob([(name, (n,), fan) for name, n, fan in lay], 3)
    rng = np.random.default_rng(0)
    centres = torch.linspace(0.8, params["r_cut"], RADIAL, device="cuda")
    xs, ys = [], []
    for seed in range(boxes):
        box = make_system(0, seed=seed)
        pos = (box.positions + jitter * rng.standard_normal(box.positions.shape)).astype(np.float32)
        snd, rcv, shift = B.mace_neighbor_list(pos.astype(np.float64), params["r_cut"], box.cells)
        g = MaceGraph(desc, blob, box.species, np.stack([snd, rcv]), shift, box.cells)
        eps, _ = g.energy(torch.from_numpy(pos).cuda())
        vec = pos[snd] + shift @ box.cells[0] - pos[rcv]
        r = torch.from_numpy(np.linalg.norm(vec, axis=1).astype(np.float32)).cuda()
        bumps = torch.exp(-4 * (r[:, None] - centres) ** 2)
        species = torch.from_numpy(box.species.astype(np.int64)).cuda()
        slot = torch.from_numpy(rcv.astype(np.int64)).cuda() * 2 + species[torch.from_numpy(snd.astype(np.int64)).cuda()]
        sums = torch.zeros(2 * len(pos), RADIAL, device="cuda").index_add_(0, slot, bumps)
        xs.append(torch.cat([sums.view(len(pos), -1), torch.nn.functional.one_hot(species, 2).float()], 1))
        ys.append(eps[:, None].clone())
        g.close()
    x, y = torch.cat(xs), torch.cat(ys)
    return (x - x.mean(0)) / (x.std(0) + 1e-3), (y - y.mean()) / y.std()


def init(n_in):
    gen = torch.Generator().manual_seed(1)

    def w(*shape):
        return (torch.randn(*shape, generator=gen) * shape[-2] ** -0.5).cuda()

    def z(*shape):
        return torch.zeros(*shape, device="cuda")
    return {"trunk.w": w(n_in, WIDTH), "trunk.b": z(WIDTH), "router.w": w(WIDTH, EXPERTS),
            "up.w": w(EXPERTS, WIDTH, HIDDEN), "up.b": z(EXPERTS, HIDDEN), "down.w": w(EXPERTS, HIDDEN, WIDTH),
            "down.b": z(EXPERTS, WIDTH), "read.w": w(WIDTH, 1), "read.b": z(1)}


def step(p, x, y):
    """The loss and its gradients."""
    h, zh = L.linear(x, p["trunk.w"], p["trunk.b"], act="silu", save=True)
    logits = L.linear(h, p["router.w"])
    top, expert = torch.topk(logits, TOP_K, dim=1)
    weights = torch.softmax(top, 1)
    plan = L.route(expert.int(), EXPERTS)
    rows = L.route_rows(h, plan)
    a, za = L.linear(rows, p["up.w"], p["up.b"], offsets=plan.offsets, act="silu", save=True)
    b = L.linear(a, p["down.w"], p["down.b"], offsets=plan.offsets)
    mixed = L.combine_rows(b, plan, weights)
    mixed += h
    out = L.linear(mixed, p["read.w"], p["read.b"])
    err = out - y
    g = {}
    dmixed, g["read.w"], g["read.b"] = L.linear_backward(err * (2 / len(y)), mixed, p["read.w"])
    db, dweights = L.combine_rows_backward(dmixed, b, plan, weights)
    da, g["down.w"], g["down.b"] = L.linear_backward(db, a, p["down.w"], offsets=plan.offsets)
    drows, g["up.w"], g["up.b"] = L.linear_backward(da, rows, p["up.w"], za, offsets=plan.offsets, act="silu")
    dtop = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
    dlogits = torch.zeros_like(logits).scatter_(1, expert, dtop)
    dh, g["router.w"], _ = L.linear_backward(dlogits, h, p["router.w"], bias=False)
    dh += L.route_rows_backward(drows, plan) + dmixed
    _, g["trunk.w"], g["trunk.b"] = L.linear_backward(dh, x, p["trunk.w"], zh, act="silu", need_dx=False)
    return (err * err).mean(), g


def train(steps=200, rate=0.03, momentum=0.9, log=print):
    """First and last loss."""
    x, y = teacher_data()
    p = init(x.shape[1])
    v = {k: torch.zeros_like(t) for k, t in p.items()}
    losses = []
    for i in range(steps):
        loss, g = step(p, x, y)
        decay = rate * (1 - i / steps)
        for k, t in p.items():
            v[k].mul_(momentum).add_(g[k])
            u = v[k]
            if k in MATRICES:
                m = g[k] + momentum * v[k]
                u = L.orthogonalise(m) * max(1.0, m.shape[-2] / m.shape[-1]) ** 0.5
            t.sub_(u, alpha=decay)
        if i % 20 == 0 or i == steps - 1:
            losses.append(loss.item())
            log(f"step {i:4d}  loss {losses[-1]:.4f}  (variance of the energies 1)", flush=True)
    return losses[0], losses[-1]


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
