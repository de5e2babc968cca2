"""Choice of experts against an FP64 form of the definition: experts equal, weights
and the logits' gradient within FP32's roundings.

Bounds: a score is the exponential of a difference of logits (rounded, 2^-24 of
its size, in the exponent) over a sum of at most 512 of them: r = (experts + 16 + 2
range) 2^-24 relative, range the largest difference of logits."""
import numpy as np
import pytest
import torch

from dense_common import DTYPES, TINY, U, U32

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def oracle(logits, k, bias, scores, groups, top_groups, normalise, scale):
    """expert, weights, scores of all experts, masks; logits float64 with -inf masked."""
    n, e = logits.shape
    live = logits > -np.inf
    l = np.where(live, logits, -np.inf)
    if scores == "sigmoid":
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-l))
    else:
        top = l.max(1, keepdims=True)
        x = np.exp(l - np.where(top > -np.inf, top, 0))
        s = x / np.maximum(x.sum(1, keepdims=True), 1e-300)
    expert, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    for t in range(n):
        c = np.where(live[t], s[t] + (0 if bias is None else bias), -np.inf)
        on = c > -np.inf
        if groups > 1:
            g = c.reshape(groups, -1)
            best = -np.sort(-g, axis=1)[:, :2]
            total = np.where(best[:, 0] > -np.inf, np.where(best > -np.inf, best, 0).sum(1), -np.inf)
            keep = np.zeros(groups, bool)
            keep[np.argsort(-total, kind="stable")[:top_groups]] = True
            on &= np.repeat(keep, e // groups)
        key = np.where(on, c if bias is not None else l[t], -np.inf)
        order = np.argsort(-key, kind="stable")[:k]
        order = order[on[order]]
        expert[t, :len(order)] = order
        v = s[t, order]
        weights[t, :len(order)] = scale * (v / v.sum() if normalise and len(v) else v)
    return expert, weights, s, live


def oracle_gradient(dw, logits, s, expert, scores, normalise, scale):
    """dlogits and the magnitude its errors are relative to."""
    n, e = s.shape
    d, mag = np.zeros((n, e)), np.zeros((n, e))
    for t in range(n):
        at = expert[t][expert[t] >= 0]
        g = dw[t][expert[t] >= 0].astype(np.float64) * scale
        v = s[t, at] / s[t, at].sum() if normalise and len(at) else s[t, at]
        with np.errstate(over="ignore"):
            one = 1 / (1 + np.exp(logits[t, at])) if scores == "sigmoid" else 1.0   # 1 - s without its cancellation
        inner, size = (g * v).sum(), (abs(g) * v).sum()
        if normalise:
            d[t, at] = v * (g - inner) * one
            mag[t, at] = v * (abs(g) + size) * one
        else:
            d[t, at], mag[t, at] = v * g * one, v * abs(g) * one
            if scores == "softmax":
                d[t] -= s[t] * inner
                mag[t] += s[t] * size
    return d, mag


def inputs(n, e, k, dtype, seed, masked=0.0, bias=False, spread=1.5):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, e, generator=gen) * spread).to(DTYPES[dtype])
    if masked:
        gone = torch.rand(n, e, generator=gen) < masked
        gone[0] = True
        x[gone] = -float("inf")
        x[1:2] = torch.finfo(x.dtype).min   # the type's lowest value masks too
        if n > 2 and e > 1:
            x[2] = -float("inf")
            x[2, e - 1] = 0.25   # one expert left
    b = torch.randn(e, generator=gen) * 0.1 if bias else None
    return x, b, torch.randn(n, k, generator=gen)


def exact_logits(x):
    v = x.double().numpy().copy()
    v[v <= torch.finfo(x.dtype).min] = -np.inf
    return v


def check(x, b, dw, k, scores="softmax", groups=1, top_groups=None, normalise=True, scale=1.0, device_x=None):
    e = x.shape[1]
    xd = x.cuda() if device_x is None else device_x
    got = L.choose_experts(xd, k, bias=None if b is None else b.cuda(), scores=scores, groups=groups, top_groups=top_groups,
                           normalise=normalise, scale=scale)
    l = exact_logits(x)
    expert, weights, s, live = oracle(l, k, None if b is None else b.double().numpy(), scores, groups, top_groups or groups,
                                      normalise, scale)
    assert np.array_equal(got.expert.cpu().numpy(), expert)
    finite = np.where(live, l, 0)
    r = (e + 16 + 2 * (finite.max(1) - finite.min(1) if x.numel() else 0)) * U32
    r = (r + 2 * abs(finite).max(1) * U32)[:, None] if x.numel() else r
    err = abs(got.weights.cpu().double().numpy() - weights) - 2 * r * abs(weights) - 2.0 ** -126
    assert not (err > 0).any(), ("weights", err.max())
    back = L.choose_experts_backward(dw.cuda(), xd, got.expert, scores=scores, normalise=normalise, scale=scale)
    assert back.dtype is x.dtype
    dw_on = np.where(expert >= 0, dw.numpy(), 0)
    s_all = s if b is None else oracle(l, k, None, scores, 1, 1, normalise, scale)[2]
    want, mag = oracle_gradient(dw_on, l, s_all, expert, scores, normalise, scale)
    name = {v: q for q, v in DTYPES.items()}[x.dtype]
    err = abs(back.cpu().double().numpy() - want) - 4 * r * mag - U[name] * abs(want) * (1 + 8 * r) - 4 * r * U[name] * mag - TINY[name]
    assert not (err > 0).any(), ("dlogits", err.max())
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("n,e,k,masked,bias", [(1, 1, 1, 0.0, False), (1, 8, 2, 0.0, True), (5, 2, 2, 0.3, False),
                                               (33, 7, 3, 0.2, True), (64, 64, 8, 0.0, False), (70, 65, 9, 0.5, True),
                                               (41, 128, 16, 0.1, True), (9, 300, 64, 0.9, False), (17, 512, 5, 0.1, True),
                                               (130, 3, 1, 0.0, True), (19, 16, 16, 0.4, True), (21, 200, 1, 0.0, False)])
def test_plain(n, e, k, masked, bias, normalise, scores, dtype):
    check(*inputs(n, e, k, dtype, n + e, masked, bias), k, scores, normalise=normalise, scale=2.5 if k > 1 else 1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("n,e,k,groups,top_groups,masked", [(40, 8, 2, 4, 1, 0.0), (64, 256, 8, 8, 4, 0.0), (33, 64, 6, 64, 9, 0.3),
                                                            (50, 35, 4, 5, 2, 0.6), (20, 512, 16, 2, 1, 0.1), (31, 6, 6, 3, 3, 0.5),
                                                            (25, 512, 3, 64, 1, 0.9)])
def test_groups(n, e, k, groups, top_groups, masked, bias, scores, dtype):
    check(*inputs(n, e, k, dtype, n + e, masked, bias), k, scores, groups, top_groups)


def test_many_rows():
    check(*inputs(3001, 256, 8, "fp32", 1, bias=True), 8, "sigmoid", 8, 4, scale=2.5)
    check(*inputs(5003, 37, 3, "bf16", 2, 0.1), 3, normalise=False)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_equal_experts_go_by_index(scores):
    x = torch.zeros(70, 100)
    x[:, 50:] = 1
    got = check(x, None, torch.randn(70, 10), 10, scores)
    assert (got.expert.cpu() == torch.arange(50, 60)).all()
    got = check(x[:, :64] * 0, torch.zeros(64), torch.randn(70, 5), 5, scores, 8, 3)
    assert (got.expert.cpu() == torch.arange(5)).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_scores_closer_than_their_roundings(scores, groups):
    """Biases that offset the scores to within FP32's roundings of a common value: the
    order is that of the FP64 sums."""
    gen = torch.Generator().manual_seed(4)
    e = 64
    x = torch.randn(1, e, generator=gen)
    s = (1 / (1 + torch.exp(-x.double())) if scores == "sigmoid" else torch.softmax(x.double(), 1))[0]
    b = (0.75 - s).float()   # s + b = 0.75 up to the rounding of b
    check(x.expand(50, e).contiguous(), b, torch.randn(50, 8, generator=gen), 8, scores, groups, max(1, groups // 2))


@pytest.mark.parametrize("e,groups,top_groups", [(35, 5, 2), (120, 8, 3), (60, 12, 5), (511, 7, 3)])
def test_rows_that_need_another_decision_among_others(e, groups, top_groups):
    """Groups that are not whole lanes, every third token with scores that only FP64 tells apart: the
    waves of a block take different ways and different times."""
    gen = torch.Generator().manual_seed(e)
    x = torch.randn(1500, e, generator=gen)
    s = 1 / (1 + torch.exp(-x[0].double()))
    b = (0.75 - s).float()
    x[::3] = x[0]   # s + b = 0.75 up to the rounding of b
    check(x, b, torch.randn(1500, 4, generator=gen), 4, "sigmoid", groups, top_groups)


def test_groups_of_large_biases_that_cancel():
    """Groups of two experts with biases c and -c: their totals are the scores' sums, which FP32 loses
    (a unit of 2^20 is 2^-4), and FP64 keeps to 2^-32."""
    x, _, dw = inputs(200, 16, 3, "fp32", 12)
    b = torch.tensor([2.0 ** 20, -2.0 ** 20] * 8)
    for scores in ("softmax", "sigmoid"):
        check(x, b, dw, 3, scores, 8, 2)


@pytest.mark.parametrize("spread", [30.0, 300.0, 3000.0])
@pytest.mark.parametrize("normalise", [True, False])
def test_large_logits(spread, normalise):
    for scores in ("softmax", "sigmoid"):
        check(*inputs(60, 40, 4, "fp32", 7, spread=spread), 4, scores, normalise=normalise)
    got = L.choose_experts(torch.full((3, 8), -500.0, device="cuda"), 4, scores="sigmoid")   # no 0 / 0
    assert torch.equal(got.weights, torch.full((3, 4), 0.25, device="cuda"))


def test_rows_without_order():
    """A NaN, or a softmax's infinity, gives valid experts and NaN weights in its row alone."""
    x, b, _ = inputs(9, 20, 3, "fp32", 3, bias=True)
    bad = x.clone()
    bad[4, 7] = float("nan")
    bad[6, 2] = float("inf")
    for scores, rows in (("softmax", [4, 6]), ("sigmoid", [4])):
        for bias in (None, b.cuda()):
            got = L.choose_experts(bad.cuda(), 3, bias=bias, scores=scores)
            keep = [i for i in range(9) if i not in rows and i != 6]
            for i in rows:
                assert got.expert[i].tolist() == [0, 1, 2] and torch.isnan(got.weights[i]).all()
            want = L.choose_experts(x.cuda(), 3, bias=bias, scores=scores)
            assert torch.equal(got.expert[keep], want.expert[keep]) and torch.equal(got.weights[keep], want.weights[keep])
    got = L.choose_experts(bad.cuda(), 3, scores="sigmoid", normalise=False)   # an infinite logit scores 1
    assert got.expert[6, 0] == 2 and got.weights[6, 0] == 1
    got = L.choose_experts(x.cuda(), 3, bias=torch.full((20,), float("nan"), device="cuda"))
    assert torch.isnan(got.weights).all() and (got.expert.cpu() == torch.arange(3)).all()


def test_infinite_biases():
    x, b, dw = inputs(50, 24, 4, "fp32", 5, bias=True)
    b[3] = b[17] = -float("inf")   # experts out of service
    got = check(x, b, dw, 4, "sigmoid")
    assert not ((got.expert == 3) | (got.expert == 17)).any()
    b[20] = float("inf")           # one that every token goes to
    got = check(x, b, dw, 4, "softmax", 4, 2)
    assert (got.expert[:, 0] == 20).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_strided_logits_and_expanded_gradients(dtype):
    x, b, dw = inputs(45, 30, 4, dtype, 9, bias=True)
    buf = torch.full((45, 41), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = buf[:, 5:35].copy_(x)
    got = check(x, b, dw, 4, device_x=view)
    one = torch.ones(1, 1, device="cuda").expand(45, 4)
    a = L.choose_experts_backward(one, view, got.expert)
    assert torch.equal(a, L.choose_experts_backward(one.contiguous(), x.cuda(), got.expert))


def test_no_tokens():
    got = L.choose_experts(torch.empty(0, 8, device="cuda"), 2)
    assert got.expert.shape == got.weights.shape == (0, 2)
    assert L.choose_experts_backward(got.weights, torch.empty(0, 8, device="cuda"), got.expert).shape == (0, 8)


def test_experts_out_of_range_take_no_part():
    x, _, dw = inputs(40, 12, 3, "fp32", 6)
    xd, dwd = x.cuda(), dw.cuda()
    e = L.choose_experts(xd, 3).expert
    e[:, 2] = torch.where(torch.arange(40, device="cuda") % 2 == 0, 12, -(1 << 31)).int()
    got = L.choose_experts_backward(dwd, xd, e)
    assert torch.equal(got, L.choose_experts_backward(dwd[:, :2].contiguous(), xd, e[:, :2].contiguous()))


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [True, False])
def test_an_expert_named_twice_gets_both_terms(scores, normalise):
    """dlogits of sum_j g_j w_j by FP64 autograd, with the scores of the experts as named."""
    gen = torch.Generator().manual_seed(11)
    x, dw = torch.randn(33, 40, generator=gen), torch.randn(33, 6, generator=gen)
    expert = torch.randint(0, 5, (33, 6), generator=gen, dtype=torch.int32)
    expert[0] = 7
    l = x.double().requires_grad_()
    s = (torch.sigmoid(l) if scores == "sigmoid" else torch.softmax(l, 1)).gather(1, expert.long())
    w = s / s.sum(1, keepdim=True) if normalise else s
    (w * dw.double()).sum().backward()
    got = L.choose_experts_backward(dw.cuda(), x.cuda(), expert.cuda(), scores=scores, normalise=normalise)
    assert torch.equal(got, L.choose_experts_backward(dw.cuda(), x.cuda(), expert.cuda(), scores=scores, normalise=normalise))
    size = (w.detach() * (dw.double().abs() + (w.detach() * dw.double().abs()).sum(1, keepdim=True))).sum(1, keepdim=True)
    assert ((got.cpu().double() - l.grad).abs() <= 4 * (40 + 16 + 20) * U32 * size).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(scores, normalise):
    """Central differences of sum(c w) along a random direction, with the experts held:
    h = 2^-7 leaves rounding (12 experts, 2^-24 * 40 / h) and truncation (h^2 / 6 times third
    derivatives below 2) under 1e-3 of the terms' size."""
    gen = torch.Generator().manual_seed(8)
    x, v = torch.randn(30, 12, generator=gen) * 2, torch.randn(30, 12, generator=gen)
    x = (x * 64).round() / 64
    c = torch.randn(30, 4, generator=gen).cuda()
    base = L.choose_experts(x.cuda(), 4, scores=scores, normalise=normalise)
    d = L.choose_experts_backward(c, x.cuda(), base.expert, scores=scores, normalise=normalise)
    h = 2.0 ** -7

    def loss(shift):
        got = L.choose_experts((x + shift * v).cuda(), 12, scores=scores, normalise=False)
        s = torch.zeros(30, 12, device="cuda", dtype=torch.float64).scatter_(1, got.expert.long(), got.weights.double())
        w = s.gather(1, base.expert.long())
        if normalise:
            w = w / w.sum(1, keepdim=True)
        return (w * c.double()).sum(1)
    want = (loss(h) - loss(-h)) / (2 * h)
    terms = (d.double() * v.cuda().double())
    assert ((terms.sum(1) - want).abs() <= 1e-3 * (terms.abs().sum(1) + c.double().abs().sum(1))).all()


def test_other_stream_and_graph():
    x, b, dw = (t.cuda() for t in inputs(4000, 96, 6, "bf16", 2, 0.1, True))

    def step(stream=None):
        c = L.choose_experts(x, 6, bias=b, groups=4, top_groups=2, stream=stream)
        return (*c, L.choose_experts_backward(dw, x, c.expert, stream=stream), *L.route(c.expert, 96, stream=stream))
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(3):
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_beyond_32_bits():
    n, e = (1 << 23) + 100, 260
    x = torch.zeros(n, e, dtype=torch.bfloat16, device="cuda")
    x[-40:] = torch.randn(40, e, device="cuda").bfloat16()
    got = L.choose_experts(x, 2)
    want = L.choose_experts(x[-40:].contiguous(), 2)
    assert torch.equal(got.expert[-40:], want.expert) and torch.equal(got.weights[-40:], want.weights)
    assert (got.expert[:-40] == torch.arange(2, device="cuda", dtype=torch.int32)).all()
    dw = torch.ones(n, 2, device="cuda")
    dw[:, 1] = 3
    d = L.choose_experts_backward(dw, x, got.expert)
    assert torch.equal(d[-40:], L.choose_experts_backward(dw[-40:].contiguous(), x[-40:].contiguous(), want.expert))
    assert (d[:-40, 0] == -0.5).all() and (d[:-40, 1] == 0.5).all()
