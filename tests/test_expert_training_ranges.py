"""Coefficients of the orthogonalising iteration whose iterates a kernel could not hold are refused: what float16 holds 64-fold for matrices of more than
one workgroup, what float holds the square of for small ones.  Singular values s go to s (a + b s^2 + c s^4): followed here on a grid."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

from paper_2603_19289_amd import moe_spec as M
from paper_2603_19289_amd import training as T

from .test_expert_training_refusals import muon, orthogonalise, recorded, refused  # noqa: F401

LARGE, SMALL = dict(rows=80, cols=96), dict(rows=16, cols=24, g_matrix_stride=16 * 24, out_matrix_stride=16 * 24, out_stride=24, g_stride=24)


def largest(coefficients, iterations, slack=0.0):
    """Of X, A and B, for any matrix: singular values fill [0, top], top at most 1 to begin with, and `slack` of it larger before each iteration."""
    a, b, c = coefficients
    top, most = 1.0, 0.0
    for _ in range(iterations):
        s = np.linspace(0.0, top * (1.0 + slack), 20001)
        q = np.abs(a + s * s * (b + s * s * c))
        top = float((s * q).max())
        most = max(most, float(q.max()), float(s[-1] ** 2), top)
        if most > 1e30:
            break
    return most


def test_iterates_beyond_a_type_are_refused():
    strong = (C.c_double * 3)(16.0, 0.0, 0.0)
    refused(orthogonalise(**LARGE, coefficients=strong, iterations=3), "orthogonalise", "iterates beyond 1000")
    refused(orthogonalise(**SMALL, coefficients=strong, iterations=17), "orthogonalise", "float's range")
    refused(muon(coefficients=(16.0, 0.0, 0.0), iterations=3), "muon_step", "iterates beyond 1000")
    refused(muon(tensor=dict(rows=16, cols=24), coefficients=(16.0, 0.0, 0.0), iterations=17), "muon_step", "float's range")


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are taken go on to the GPU, with addresses that are none")
def test_what_is_refused_is_what_would_not_fit():
    """A call that is taken fails for want of a GPU here.  The usual coefficients are taken, however often; where the end of the range is pushed out
    fivefold by each iteration, (0, 0, 1), the 64th for roundings comes to (65 / 64)^(5 + 25 + .. + 3125) in five."""
    def answer(kind, coefficients, iterations):
        return orthogonalise(**kind, coefficients=(C.c_double * 3)(*coefficients), iterations=iterations)
    for c in ((3.4445, -4.775, 2.0315), (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (15 / 8, -10 / 8, 3 / 8), (3.0, -3.2, 1.2), (1.0, 0.0, 0.0), (0.0, 0.0, 0.0),
              (-1.5, 0.5, 0.0)):
        for n in (1, 5, 64):
            assert answer(LARGE, c, n) == answer(SMALL, c, n) == M.EHIP, (c, n)
    assert [answer(LARGE, (0.0, 0.0, 1.0), n) for n in (1, 5)] == [M.EHIP, M.EINVAL] and answer(SMALL, (0.0, 0.0, 1.0), 5) == M.EHIP
    r, taken = random.Random(1), 0
    for _ in range(400):
        size = r.choice([1.0, 3.0, 16.0])
        c, n = tuple(r.uniform(-size, size) * r.choice([0, 1, 1, 1]) for _ in range(3)), r.choice([1, 2, 3, 5, 9, 64])
        for kind, limit, slack in ((LARGE, 1000.0, 1 / 64), (SMALL, 2.0 ** 60, 2.0 ** -18)):
            got, most = answer(kind, c, n), largest(c, n, slack)
            assert got in (M.EINVAL, M.EHIP)
            taken += got == M.EHIP
            if abs(most / limit - 1) > 0.01:          # the grid and the roots that the library takes agree
                assert (got == M.EHIP) == (most <= limit), (c, n, most)
            assert got == M.EINVAL or largest(c, n) <= limit, (c, n)
    assert 200 < taken < 700                      # both answers are given


@pytest.mark.parametrize("coefficients", [(), (1.5, -0.5), (3.4445, -4.775, 2.0315, 0.0)])
def test_the_iteration_has_three_coefficients(recorded, coefficients):  # noqa: F811
    """Two were taken as if the third were zero."""
    p = torch.zeros(70, 90)
    for call in (lambda: T.orthogonalise(p, coefficients=coefficients), lambda: T.Muon([p], lr=0.1, coefficients=coefficients)):
        with pytest.raises(ValueError, match="three"):
            call()
    opt = T.Muon([p], lr=0.1)
    opt.coefficients = coefficients                # settings may be changed between steps
    with pytest.raises(ValueError, match="three"):
        opt.step([p.clone()])
    opt.coefficients = [1.5, -0.5, 0.0]
    opt.step([p.clone()])
    assert list(recorded[-1][2]._obj.coefficients) == [1.5, -0.5, 0.0]
