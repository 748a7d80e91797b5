"""Which polynomials orthogonal updates take: bounds of singular values that the host derives, before anything reaches a device."""
import math

import numpy as np
import pytest
import torch

from paper_2103_07454_b200 import binding as B
from test_more_operators_host import A, Matrix, orthogonalise, refused, workspace


def largest(coefficients):
    """The largest singular value on the way from 0 .. 1, by sampling: step by step, of the whole range that the step before leaves."""
    top = most = 1.0
    for a, b, c in coefficients:
        top = max(abs(s * (a + b * s * s + c * s ** 4)) for s in (top * k / 20000 for k in range(20001)))
        most = max(most, top)
    return most


@pytest.mark.parametrize("c", [0.0, 1e-300, 1e-30, 1e-20, -1e-20, 1e-17, 1e-13, 1e-6, -1e-6, 1.0, -1.0])
@pytest.mark.parametrize("a,b", [(1000.0, -1000.0), (30.0, -30.0), (-30.0, 30.0), (1000.0, -999.0), (100.0, -163.0), (1.5, -0.5), (0.0, 50.0), (60.0, 0.0), (0.0, 0.0)])
def test_growth_inside_the_range_is_found(a, b, c):
    """A fifth-degree term next to nothing beside the third: what the values reach on the way counts, not where 1 ends up."""
    q = orthogonalise(coefficients=[a, b, c], steps=1)
    reach = largest([(a, b, c)])
    # the host leaves a hundredth for roundings: 64 / 1.01; samples find a maximum to 1e-8 of it
    limit = 64 / 1.01
    assert abs(reach - limit) > 0.1
    assert refused(q) if reach > limit else workspace(q) > 0


def test_the_model_of_the_growth():
    assert math.isclose(largest([(1.5, -0.5, 0.0)]), 1.0)
    assert math.isclose(largest([(30.0, -30.0, 0.0)]), 20 / math.sqrt(3), rel_tol=1e-4)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("rows,columns", [(1, 1), (64, 64), (65, 63), (1, 1 << 20), (1 << 20, 1), (64, 1 << 18), (1000, 3000), (2048, 2048), (16384, 8192)])
def test_the_workspace_is_what_the_header_says(rows, columns, dtype):
    m = dict(rows=rows, columns=columns, velocity=Matrix())
    m["grad"] = m["out"] = Matrix(A, rows * columns, columns)
    for P in (1, 3):
        values = P * (-rows % 64 + rows) * (-columns % 64 + columns)
        need = workspace(orthogonalise(matrices=[m], P=P, dtype=dtype, out_dtype=dtype))
        # (8-bit results: a float a row beside the boxes, in whole boxes; tables on boundaries of 256 bytes)
        assert 6 * values <= need <= 20 * values + 1024 * P + 3 * 256 + 8192 * P
        assert workspace(orthogonalise(matrices=[m] * 7, P=P, dtype=dtype, out_dtype=dtype)) <= max(need, 1 << 30) + 7 * 2048 * P


@pytest.mark.parametrize("scale", [1, 2.0, np.float32(0.5), np.float64(0.5), np.int64(2), [0.5], np.array([0.5]), torch.tensor([0.5])])
def test_numbers_of_any_kind_scale(scale):
    """They get as far as the tensor that is not on a device."""
    with pytest.raises(B.EventGradError, match="no CUDA device"):
        B.orthogonalise([torch.zeros(1, 4, 8)], scale=scale)


@pytest.mark.parametrize("bad", [None, "xy", 1j, np.array(0.5), torch.tensor(0.5), [0.5, 0.5], object()])
def test_other_scales_are_refused_as_other_arguments_are(bad):
    """Before anything asks for their entries."""
    with pytest.raises(B.EventGradError, match="scale"):
        B.orthogonalise([torch.zeros(1, 4, 8)], scale=bad)


@pytest.mark.parametrize("bad", [1, torch.tensor(0.5)])
def test_arguments_that_hold_nothing_are_refused_as_others_are(bad):
    for name in ("out", "velocity", "velocity_out"):
        with pytest.raises(B.EventGradError):
            B.orthogonalise([torch.zeros(1, 4, 8)], **{name: bad})
