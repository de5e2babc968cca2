"""Argument errors of the dense entry points: the documented status, before any
device work (host pointers and NULLs never reach a kernel), on the CPU."""
import copy
import os

import numpy as np
import pytest

B = pytest.importorskip("paper_2510_23621_amd.binding")
pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmace_amd.so not built")

EINVAL, ERANGE, ENOSPACE, EUNSUPPORTED = -1, -2, -3, -7
A = np.zeros(4096, np.float64)   # stands for every tensor: refused calls do not touch it


def linear_desc(**kw):
    d = dict(n_rows=10, n_in=8, n_out=16, n_groups=2, dtype=0, act=1, ld_x=8, ld_y=16, ld_residual=16, ld_preact=16)
    d.update(kw)
    return B.mace_linear_desc(**d)


BAD_LINEAR = [(dict(n_rows=-1), EINVAL), (dict(n_in=0), EINVAL), (dict(n_out=0), EINVAL), (dict(n_groups=0), EINVAL),
              (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(act=3), EINVAL), (dict(ld_x=7), EINVAL),
              (dict(ld_y=15), EINVAL), (dict(ld_residual=15), EINVAL), (dict(ld_preact=15), EINVAL),
              (dict(n_groups=1025), EUNSUPPORTED), (dict(n_rows=(1 << 30) + 1), EUNSUPPORTED),
              (dict(n_in=(1 << 20) + 1, ld_x=1 << 21), EUNSUPPORTED)]


def code(f, *a):
    return getattr(B.lib(), f)(*[x.ctypes.data if isinstance(x, np.ndarray) else x for x in a])


@pytest.mark.parametrize("change,want", BAD_LINEAR)
def test_linear_descriptor(change, want):
    d = linear_desc(**change)
    assert code("mace_linear_forward", d, A, A, A, A, A, A, A, None) == want
    assert code("mace_linear_backward_workspace_bytes", d, 1, 1) == 0
    assert code("mace_linear_backward", d, A, 16, A, A, A, A, A, 8, A, A, A, 1 << 30, None) == want


def test_linear_arguments():
    d = linear_desc()
    ok = [d, A, A, A, A, A, A, A, None]
    assert code("mace_linear_forward", None, *ok[1:]) == EINVAL
    for i in (1, 2, 5, 6):   # x, weights, offsets of two groups, y
        bad = list(ok)
        bad[i] = None
        assert code("mace_linear_forward", *bad) == EINVAL
    ok = [d, A, 16, A, A, A, A, A, 8, A, A, A, 1 << 30, None]
    for i in (1, 3, 4, 5, 6, 11):   # dy, x, weights, z of an activation, offsets, workspace
        bad = list(ok)
        bad[i] = None
        assert code("mace_linear_backward", *bad) == EINVAL
    for i, v in ((2, 15), (8, 7)):
        bad = list(ok)
        bad[i] = v
        assert code("mace_linear_backward", *bad) == EINVAL
    need = B.mace_linear_backward_workspace_bytes(d, True, True)
    assert need > 0
    assert code("mace_linear_backward", *ok[:12], 16, None) == ENOSPACE


def test_linear_without_rows_or_work_returns_ok():
    assert code("mace_linear_forward", linear_desc(n_rows=0), None, A, None, None, A, None, None, None) == 0


def route_desc(**kw):
    d = dict(n_tokens=10, top_k=2, n_experts=4, width=8, dtype=0, ld_tokens=8, ld_rows=8)
    d.update(kw)
    return B.mace_route_desc(**d)


@pytest.mark.parametrize("change,want", [
    (dict(n_tokens=-1), EINVAL), (dict(top_k=0), EINVAL), (dict(n_experts=0), EINVAL), (dict(width=0), EINVAL),
    (dict(dtype=5), EINVAL), (dict(ld_tokens=7), EINVAL), (dict(ld_rows=7), EINVAL), (dict(n_experts=513), EUNSUPPORTED),
    (dict(n_tokens=1 << 30, top_k=2), EUNSUPPORTED), (dict(width=(1 << 20) + 1, ld_tokens=1 << 21, ld_rows=1 << 21),
                                                      EUNSUPPORTED)])
def test_route_descriptor(change, want):
    d = route_desc(**change)
    assert code("mace_route_workspace_bytes", d) == 0
    assert code("mace_route_build", d, A, A, A, A, A, 1 << 30, None) == want
    assert code("mace_route_gather", d, A, A, A, A, None) == want
    assert code("mace_route_combine", d, A, A, A, A, A, None) == want
    assert code("mace_route_combine_backward", d, A, A, A, A, A, A, A, None) == want


def test_route_arguments():
    d = route_desc()
    calls = {"mace_route_build": ([d, A, A, A, A, None, 0, None], (0, 1, 2, 3, 4)),
             "mace_route_gather": ([d, A, A, A, A, None], (0, 1, 2, 3, 4)),
             "mace_route_combine": ([d, A, A, A, A, A, None], (0, 1, 3, 4, 5)),
             "mace_route_combine_backward": ([d, A, A, A, A, A, A, A, None], (0, 1, 2, 4, 5))}
    for f, (args, required) in calls.items():
        for i in required:
            bad = copy.copy(args)
            bad[i] = None
            assert code(f, *bad) == EINVAL, (f, i)
    big = route_desc(n_tokens=5000)
    assert code("mace_route_build", big, A, A, A, A, None, 0, None) == EINVAL
    assert code("mace_route_build", big, A, A, A, A, A, 16, None) == ENOSPACE


COEF = np.array([[3.4445, -4.7750, 2.0315]] * 5)


def orth_desc(**kw):
    d = dict(batch=2, rows=6, cols=9, dtype=0, n_steps=5, ld_g=9, stride_g=54, ld_out=9, stride_out=54, eps=1e-7)
    d.update(kw)
    return B.mace_orthogonalise_desc(**d)


@pytest.mark.parametrize("change,want", [
    (dict(batch=-1), EINVAL), (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(dtype=3), EINVAL),
    (dict(n_steps=-1), EINVAL), (dict(n_steps=65), EINVAL), (dict(ld_g=8), EINVAL), (dict(ld_out=8), EINVAL),
    (dict(stride_g=-1), EINVAL), (dict(stride_out=53), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(rows=(1 << 15) + 1, stride_out=1 << 40), EUNSUPPORTED),
    (dict(batch=65536), EUNSUPPORTED)])
def test_orthogonalise_descriptor(change, want):
    d = orth_desc(**change)
    assert code("mace_orthogonalise_workspace_bytes", d) == 0
    assert code("mace_orthogonalise", d, A, COEF, A, A, 1 << 30, None) == want


def test_orthogonalise_arguments():
    ok = [orth_desc(), A, COEF, A, A, 1 << 30, None]
    for i in (0, 1, 2, 3, 4):
        bad = list(ok)
        bad[i] = None
        assert code("mace_orthogonalise", *bad) == EINVAL
    assert code("mace_orthogonalise", *ok[:5], 100, None) == ENOSPACE
    assert code("mace_orthogonalise", orth_desc(batch=0), None, COEF, None, None, 0, None) == 0


@pytest.mark.parametrize("step", [(5.0, 0.0, 0.0), (1.0, 300.0, -300.0), (1.0, float("inf"), 0.0),
                                  (float("nan"), 0.0, 0.0), (3.4445, -4.775, 20.0)])
def test_orthogonalise_refuses_steps_out_of_range(step):
    """A step that could take a singular value past 3.4, or b A + c A A past 200."""
    coef = np.array([[1.5, -0.5, 0.0]] * 4 + [list(step)])
    assert code("mace_orthogonalise", orth_desc(), A, coef, A, A, 1 << 30, None) == ERANGE


def test_layers_refuse_before_the_library():
    import torch

    from paper_2510_23621_amd import layers
    x = torch.zeros(4, 8)
    for f in (lambda: layers.linear(x, torch.zeros(8, 8)), lambda: layers.route(torch.zeros(4, 1, dtype=torch.int32), 2),
              lambda: layers.orthogonalise(x)):
        with pytest.raises(ValueError):   # host tensors
            f()
