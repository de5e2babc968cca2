"""What layers.py does around the calls of embeddings, the choice of experts and the
8-bit layers, on the CPU: refusals of tensors that do not fit, devices and streams,
gradients that would be lost, sizes that 32 bits cannot hold."""
import pytest
import torch

from test_layers_calls import Stream, machine  # noqa: F401

L = pytest.importorskip("paper_2510_23621_amd.layers")
F, I, Q = torch.float32, torch.int32, torch.int8


def calls(device, **kw):
    def t(*shape, dtype=F):
        return torch.empty(*shape, dtype=dtype, device=device)
    rows = L.Rows8(t(6, 16, dtype=Q), t(6), 8)
    z = L.Rows8(t(6, 16, dtype=Q), t(6), 4)
    w8 = L.Weights8(t(1, 4, 16, dtype=Q), t(1, 4), 8)
    return {"embed": lambda: L.embed(t(6, dtype=I), t(5, 8), **kw),
            "embed_backward": lambda: L.embed_backward(t(6, 8), t(6, dtype=I), 5, **kw),
            "choose_experts": lambda: L.choose_experts(t(6, 8), 2, bias=t(8), **kw),
            "choose_experts_backward": lambda: L.choose_experts_backward(t(6, 2), t(6, 8), t(6, 2, dtype=I), **kw),
            "pack_rows": lambda: L.pack_rows(t(6, 8), **kw), "unpack_rows": lambda: L.unpack_rows(rows, **kw),
            "pack_weights": lambda: L.pack_weights(t(8, 4), **kw), "linear8": lambda: L.linear8(t(6, 8), w8, **kw),
            "linear8 of rows": lambda: L.linear8(rows, w8, act="silu", **kw),
            "linear8 by name": lambda: L.linear8(w=w8, x=rows, **kw),
            "linear_backward8": lambda: L.linear_backward8(t(6, 4), rows, t(8, 4), z, act="gelu", **kw)}


NAMES = list(calls("cpu"))


@pytest.mark.parametrize("name", NAMES)
def test_the_tensors_device_is_current_for_the_call(machine, name):  # noqa: F811
    for index in (0, 1, 3):
        machine.calls.clear()
        calls(f"cuda:{index}")[name]()
        assert [c[1] for c in machine.calls] == [index] and machine.current == 0
        assert machine.calls[0][2][-1] == 1000 + index


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(machine, name):  # noqa: F811
    calls("cuda:1", stream=Stream(1))[name]()
    assert [c[1] for c in machine.calls] == [1] and machine.current == 0
    machine.calls.clear()
    with pytest.raises(ValueError, match="stream"):
        calls("cuda:1", stream=Stream(0))[name]()
    assert not machine.calls and machine.current == 0


def t(*shape, dtype=F, device="cuda:0"):
    return torch.empty(*shape, dtype=dtype, device=device)


def rows8(n=6, columns=8, padded=16, device="cuda:0"):
    return L.Rows8(t(n, padded, dtype=Q, device=device), t(n, device=device), columns)


def weights8(g=1, m=4, k=8, padded=16, device="cuda:0"):
    return L.Weights8(t(g, m, padded, dtype=Q, device=device), t(g, m, device=device), k)


OTHER = "cuda:1"
REFUSED = [
    lambda: L.embed(t(6, dtype=torch.int64), t(5, 8)), lambda: L.embed(t(6, dtype=I), t(5, 8, device=OTHER)),
    lambda: L.embed(t(6, dtype=I), t(5, 8, dtype=torch.float64)), lambda: L.embed(t(6, dtype=I), t(8, 5).t()),
    lambda: L.embed(t(6, 2, dtype=I)[:, 0], t(5, 8)), lambda: L.embed(t(6, dtype=I), t(5, 2, 8)),
    lambda: L.embed_backward(t(6, 8), t(7, dtype=I), 5), lambda: L.embed_backward(t(6, 8), t(6, dtype=I), 0),
    lambda: L.embed_backward(t(6, 8), t(6, dtype=I), 1 << 31), lambda: L.embed_backward(t(6, 8, device=OTHER), t(6, dtype=I), 5),
    lambda: L.embed_backward(t(6, 8, dtype=torch.float64), t(6, dtype=I), 5),
    lambda: L.embed(t(1, dtype=I), t(4, 2 ** 32 + 8)), lambda: L.embed_backward(t(1, 2 ** 32 + 8), t(1, dtype=I), 5),
    lambda: L.choose_experts(t(6, 8), 2, scores="cosine"), lambda: L.choose_experts(t(6, 8), 0),
    lambda: L.choose_experts(t(6, 8), 2 ** 32 + 2), lambda: L.choose_experts(t(6, 8), 2, groups=2 ** 32 + 2),
    lambda: L.choose_experts(t(6, 8), 2, groups=4, top_groups=0), lambda: L.choose_experts(t(6, 8), 2, bias=t(7)),
    lambda: L.choose_experts(t(6, 8), 2, bias=t(8, dtype=torch.bfloat16)), lambda: L.choose_experts(t(6, 8), 2, bias=t(8, device=OTHER)),
    lambda: L.choose_experts(t(6, 8, dtype=torch.float64), 2), lambda: L.choose_experts(t(8, 6).t(), 2),
    lambda: L.choose_experts(t(1, 2 ** 32 + 8), 2),
    lambda: L.choose_experts_backward(t(6, 3), t(6, 8), t(6, 2, dtype=I)),
    lambda: L.choose_experts_backward(t(6, 2, dtype=torch.bfloat16), t(6, 8), t(6, 2, dtype=I)),
    lambda: L.choose_experts_backward(t(6, 2), t(5, 8), t(6, 2, dtype=I)),
    lambda: L.choose_experts_backward(t(6, 2), t(6, 8), t(6, 2, dtype=torch.int64)),
    lambda: L.choose_experts_backward(t(6, 2), t(6, 8), t(6, 2, dtype=I, device=OTHER)),
    lambda: L.choose_experts_backward(t(6, 2), t(6, 8, device=OTHER), t(6, 2, dtype=I)),
    lambda: L.pack_rows(t(6, 8, dtype=torch.float64)), lambda: L.pack_rows(t(8, 6).t()), lambda: L.pack_rows(t(1, 2 ** 32 + 8)),
    lambda: L.unpack_rows(rows8(), torch.int8), lambda: L.unpack_rows(rows8(columns=17)), lambda: L.unpack_rows(rows8(columns=0)),
    lambda: L.unpack_rows(rows8()._replace(scales=t(5))), lambda: L.unpack_rows(rows8()._replace(scales=t(6, device=OTHER))),
    lambda: L.unpack_rows(rows8()._replace(values=t(6, 16))), lambda: L.unpack_rows(rows8()._replace(values=t(16, 6, dtype=Q).t())),
    lambda: L.pack_weights(t(8, 4, dtype=torch.float64)), lambda: L.pack_weights(t(4, 8).t()), lambda: L.pack_weights(t(8)),
    lambda: L.pack_weights(t(1, 1, 2 ** 32 + 8)),
    lambda: L.linear8(t(6, 8), weights8(), act="relu"), lambda: L.linear8(t(6, 9), weights8()), lambda: L.linear8(t(6, 8), weights8(g=2)),
    lambda: L.linear8(t(6, 8), weights8(device=OTHER)), lambda: L.linear8(t(6, 8), weights8()._replace(scales=t(1, 5))),
    lambda: L.linear8(t(6, 8), weights8()._replace(values=t(1, 4, 16))), lambda: L.linear8(t(6, 8), weights8(k=17)),
    lambda: L.linear8(t(6, 8), weights8(), t(5)), lambda: L.linear8(t(6, 8), weights8(), t(4, dtype=torch.bfloat16)),
    lambda: L.linear8(t(6, 8), weights8(), None, t(6, 5)), lambda: L.linear8(t(6, 8), weights8(), dtype=torch.bfloat16),
    lambda: L.linear8(t(6, 8), weights8(g=2), offsets=t(2, dtype=I)), lambda: L.linear8(t(6, 8), weights8(g=2), t(4), offsets=t(3, dtype=I)),
    lambda: L.linear8(rows8(), weights8(), dtype=torch.int8), lambda: L.linear8(rows8(), weights8(), t(4), dtype=torch.bfloat16),
    lambda: L.linear8(rows8(), weights8(), None, t(6, 4, dtype=torch.bfloat16)), lambda: L.linear8(rows8(columns=9), weights8()),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4), act="relu"), lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4), act="silu"),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(9, 4)), lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 5)),
    lambda: L.linear_backward8(t(6, 4), rows8(n=5), t(8, 4)), lambda: L.linear_backward8(t(6, 4), rows8(), t(4, 8).t()),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4, dtype=torch.bfloat16)), lambda: L.linear_backward8(t(6, 4), rows8(device=OTHER), t(8, 4)),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4, device=OTHER)), lambda: L.linear_backward8(t(6, 4), rows8(), t(2, 8, 4)),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4), rows8(columns=5), act="silu"),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4), rows8(n=7, columns=4), act="silu"),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(8, 4), rows8(columns=4, device=OTHER), act="silu"),
    lambda: L.linear_backward8(t(6, 4), rows8(), t(2, 8, 4), offsets=t(2, dtype=I))]


@pytest.mark.parametrize("call", range(len(REFUSED)))
def test_refused(machine, call):  # noqa: F811
    with pytest.raises(ValueError):
        REFUSED[call]()
    assert not machine.calls


def g(*shape, dtype=F):
    return torch.zeros(*shape, dtype=dtype, requires_grad=True)


def c(*shape, dtype=F):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("call", [
    lambda: L.embed(c(4, dtype=I), g(5, 8)), lambda: L.embed_backward(g(4, 8), c(4, dtype=I), 5), lambda: L.choose_experts(g(4, 8), 2),
    lambda: L.choose_experts(c(4, 8), 2, bias=g(8)), lambda: L.choose_experts_backward(g(4, 2), c(4, 8), c(4, 2, dtype=I)),
    lambda: L.pack_rows(g(4, 8)), lambda: L.pack_weights(g(8, 4)), lambda: L.unpack_rows(L.Rows8(c(4, 16, dtype=Q), g(4), 8)),
    lambda: L.linear8(g(4, 8), L.Weights8(c(1, 4, 16, dtype=Q), c(1, 4), 8)),
    lambda: L.linear8(c(4, 8), L.Weights8(c(1, 4, 16, dtype=Q), g(1, 4), 8)),
    lambda: L.linear_backward8(c(4, 4), L.Rows8(c(4, 16, dtype=Q), c(4), 8), g(8, 4))])
def test_refused_while_gradients_are_recorded(call):
    with pytest.raises(ValueError, match="no_grad"):
        call()
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):   # (then the host tensors are what is wrong)
        call()


def test_host_tensors_are_refused():
    for name, call in calls("cpu").items():
        with pytest.raises(ValueError, match="GPU"):
            call()
