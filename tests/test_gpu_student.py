"""Embedding, choice of experts, routing and expert layers together, as a program uses
them: the gradients of a training step against FP64 autograd at the choice it made,
and the served form against its own definition, eager and captured."""
import os
import sys

import pytest
import torch

from dense_common import U32

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
L = pytest.importorskip("paper_2510_23621_amd.layers")
N, SPECIES, D, H, E, K = 700, 9, 40, 56, 12, 3


def parameters(seed=0):
    gen = torch.Generator().manual_seed(seed)
    return {"table": torch.randn(SPECIES, D, generator=gen), "router": torch.randn(D, E, generator=gen) * D ** -0.5,
            "up": torch.randn(E, D, H, generator=gen) * D ** -0.5, "up_b": torch.randn(E, H, generator=gen) * 0.3,
            "down": torch.randn(E, H, D, generator=gen) * H ** -0.5}


def data(seed=1):
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, SPECIES, (N,), generator=gen, dtype=torch.int32)
    ids[::11] = -1
    return ids, torch.randn(N, D, generator=gen), torch.randn(N, D, generator=gen) * 0.1, torch.randn(E, generator=gen) * 0.05


def step(p, ids, x, dout, b, keep8, stream=None):
    """Output, choice and gradients of h = x + embed(ids), out = sum_j w_j down(silu(up(h)))."""
    kw = {"stream": stream}
    h = L.embed(ids, p["table"], scale=2.0, **kw)
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        h = h + x
    logits = L.linear(h, p["router"], **kw)
    how = dict(scores="sigmoid", scale=1.5)
    c = L.choose_experts(logits, K, bias=b, groups=4, top_groups=2, **how, **kw)
    plan = L.route(c.expert, E, **kw)
    rows = L.route_rows(h, plan, **kw)
    a, z = L.linear(rows, p["up"], p["up_b"], offsets=plan.offsets, act="silu", save=True, **kw)
    y = L.linear(a, p["down"], offsets=plan.offsets, **kw)
    out = L.combine_rows(y, plan, c.weights, **kw)
    dy, dw = L.combine_rows_backward(dout, y, plan, c.weights, **kw)
    da, ddown, _ = L.linear_backward(dy, a, p["down"], offsets=plan.offsets, bias=False, **kw)
    if keep8:
        drows, dup, dup_b = L.linear_backward8(da, L.pack_rows(rows, **kw), p["up"], L.pack_rows(z, **kw), offsets=plan.offsets,
                                               act="silu", **kw)
    else:
        drows, dup, dup_b = L.linear_backward(da, rows, p["up"], z, offsets=plan.offsets, act="silu", **kw)
    dlogits = L.choose_experts_backward(dw, logits, c.expert, **how, **kw)
    dh, drouter, _ = L.linear_backward(dlogits, h, p["router"], bias=False, **kw)
    back = L.route_rows_backward(drows, plan, **kw)
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        dh = dh + back
    dtable = L.embed_backward(dh, ids, SPECIES, scale=2.0, **kw)
    return {"out": out, "expert": c.expert, "table": dtable, "router": drouter, "up": dup, "up_b": dup_b, "down": ddown}


def oracle(p, ids, x, dout, expert):
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    on = (ids >= 0)[:, None]
    h = x.double() + torch.where(on, 2.0 * q["table"][ids.clamp_min(0).long()], 0.0)
    s = torch.sigmoid(h @ q["router"]).gather(1, expert.long())
    w = 1.5 * s / s.sum(1, keepdim=True)
    out = torch.zeros(N, D, dtype=torch.float64)
    for j in range(K):
        for e in range(E):
            at = torch.nonzero(expert[:, j] == e)[:, 0]
            z = h[at] @ q["up"][e] + q["up_b"][e]
            out = out.index_add(0, at, w[at, j, None] * (z * torch.sigmoid(z) @ q["down"][e]))
    (out * dout.double()).sum().backward()
    return {"out": out.detach()} | {k: v.grad for k, v in q.items()}


@pytest.mark.parametrize("keep8", [False, True])
def test_step_against_autograd(keep8):
    """FP32: 400 roundings' worth of the largest entry (chains of sums of up to 700 terms whose
    errors add in squares). Kept in 8 bits, x and z are off by at most 1/254 of their row's
    largest magnitude: up to 2 % of the up layer's and its inputs' gradients in the norm."""
    p, (ids, x, dout, b) = parameters(), data()
    got = step({k: v.cuda() for k, v in p.items()}, ids.cuda(), x.cuda(), dout.cuda(), b.cuda(), keep8)
    want = oracle(p, ids, x, dout, got["expert"].cpu())
    for k, v in want.items():
        err = (got[k].cpu().double() - v)
        if keep8 and k in ("table", "router", "up", "up_b"):
            assert err.norm() <= 0.02 * v.norm(), k
        else:
            assert err.abs().max() <= 400 * U32 * v.abs().max(), (k, err.abs().max() / v.abs().max())


@pytest.mark.parametrize("keep8", [False, True])
def test_step_captured_and_on_another_stream(keep8):
    p, args = {k: v.cuda() for k, v in parameters().items()}, [t.cuda() for t in data()]
    want = step(p, *args, keep8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(p, *args, keep8, stream=s)
    s.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(p, *args, keep8)
    fresh = data(7)
    for source in (fresh, data(), fresh):   # new inputs in the captured buffers
        for a, t in zip(args, source):
            a.copy_(t)
        for t in out.values():
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = step(p, *args, keep8)
        assert all(torch.equal(out[k], want[k]) for k in want)


def test_two_graphs_at_once():
    """Two captured steps hold workspaces of their own: replayed on two streams together
    they give what they give alone."""
    p = {k: v.cuda() for k, v in parameters().items()}
    sets = [[t.cuda() for t in data(i)] for i in (1, 2)]
    graphs, outs = [], []
    for a in sets:
        step(p, *a, True)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(p, *a, True))
        graphs.append(g)
    want = [step(p, *a, True) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(o[k], w[k]) for k in w)


@pytest.mark.parametrize("n", [1, 5, 700])
def test_served_in_8_bits(n):
    """The served layers are linear at the values that the 8-bit rows and weights stand for: each
    checked on the input it got, to FP32's roundings."""
    p, (ids, x, _, b) = {k: v.cuda() for k, v in parameters().items()}, [t.cuda() for t in data()]
    up, down = L.pack_weights(p["up"]), L.pack_weights(p["down"])
    h = x[:n] + L.embed(ids[:n], p["table"])
    c = L.choose_experts(L.linear(h, p["router"]), K, bias=b)
    plan = L.route(c.expert, E)
    rows = L.route_rows(h, plan)

    def stands(w, k):
        return (w.values.double() * w.scales.double()[..., None])[..., :k].transpose(1, 2).cpu()

    def check(x8, w, bias, got, act):
        at = (x8.values.double() * x8.scales.double()[:, None])[:, :x8.columns].cpu()
        off, W = plan.offsets.tolist(), stands(w, x8.columns)
        for e in range(E):
            a = at[off[e]:off[e + 1]]
            z = a @ W[e] + (bias[e].cpu().double() if bias is not None else 0)
            y = z * torch.sigmoid(z) if act else z
            err = (got[off[e]:off[e + 1]].cpu().double() - y).abs()
            assert (err <= 40 * U32 * (1 + a.abs() @ W[e].abs())).all()
    a = L.linear8(rows, up, p["up_b"], offsets=plan.offsets, act="silu")
    check(L.pack_rows(rows), up, p["up_b"], a, True)
    y = L.linear8(a, down, offsets=plan.offsets)
    check(L.pack_rows(a), down, None, y, False)
    assert torch.isfinite(L.combine_rows(y, plan, c.weights)).all()


def test_example_keeps_activations_in_8_bits_and_serves():
    """Gradients of the step with 8-bit activations point where the FP32 ones do (their rows are off
    by at most 1/254 of the largest entry: 2 % in the norm), and serving runs."""
    import distil_head as D_
    gen = torch.Generator().manual_seed(3)
    x, y = torch.randn(200, 20, generator=gen).cuda(), torch.randn(200, 1, generator=gen).cuda()
    p = D_.init(20)
    loss, g = D_.step(p, x, y)
    loss8, g8 = D_.step(p, x, y, keep8=True)
    assert torch.equal(loss, loss8)
    for k in g:
        assert (g[k] - g8[k]).norm() <= 0.02 * g[k].norm(), k
    out = D_.predict(D_.serve(p), x)
    assert out.shape == y.shape and torch.isfinite(out).all()
    D_.train(3, log=lambda *a, **k: None, keep8=True)
