"""The steps that `orthogonalise` hands to the library: any sequence of triples, read
anew in every call; anything else is refused."""
import ctypes

import numpy as np
import pytest

from test_layers_calls import machine, tensors  # noqa: F401

L = pytest.importorskip("paper_2510_23621_amd.layers")
STEPS = [[1.5, -0.5, 0.0], [3.0, -3.2, 1.2]]


@pytest.fixture
def handed(machine):  # noqa: F811
    """The steps that the library gets."""
    g = tensors("cuda:0")[0]

    def call(coefficients):
        got = []

        def record(d, _, coef, *args):
            got.append(np.ctypeslib.as_array(ctypes.cast(coef, ctypes.POINTER(ctypes.c_double)), (d.n_steps, 3)).tolist()
                       if d.n_steps else [])
            return 0
        machine.mace_orthogonalise = record
        L.orthogonalise(g, coefficients)
        return got[0]
    return call


def test_forms(handed):
    for c in (STEPS, tuple(map(tuple, STEPS)), tuple(STEPS), [tuple(s) for s in STEPS], np.array(STEPS)):
        assert handed(c) == STEPS
    assert handed(()) == [] and handed([]) == []
    assert handed(s for s in STEPS) == STEPS and handed(iter(STEPS)) == STEPS


def test_read_anew(handed):
    a = np.float64(1.5), np.array(-0.5), 0.0
    steps = (a,)
    assert handed(steps) == [[1.5, -0.5, 0.0]]
    a[1][...] = -0.25
    assert handed(steps) == [[1.5, -0.25, 0.0]]


@pytest.mark.parametrize("bad", [((1.5, -0.5),) * 3, ((1.5, -0.5, 0.0, 1.0),) * 3, (1.5, -0.5, 0.0), ((1.5,),) * 3,
                                 (((1.5, -0.5, 0.0),),), ((1.5, -0.5, 0.0), (1.5, -0.5))], ids=str)
def test_not_triples(handed, bad):
    with pytest.raises(ValueError, match="triples"):
        handed(bad)
