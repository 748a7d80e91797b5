"""Which polynomials orthogonal updates take: bounds of singular values that the host derives, before anything reaches a device."""
import math

import pytest

from test_more_operators_host import orthogonalise, refused, workspace


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
