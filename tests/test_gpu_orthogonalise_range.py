"""Orthogonal updates by polynomials that make values small, against the definition in 64 bits."""
import math

import pytest
import torch

import test_gpu_orthogonalise as O
from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,result", [("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32")])
@pytest.mark.parametrize("factor,steps", [(0.25, 20), (0.5, 64), (-0.7, 64), (0.25, 49), (3.0, 3)])
def test_a_factor_alone(factor, steps, dtype, result):
    """X <- factor X: results of down to 2^-98 of the gradient's direction.  Each step rounds X once (to two parts of 11 bits, 2^-23; the
    bound for 8-bit results leaves it 2^-12), the result once; `scale`, a power of two, brings them to where its type has all its bits."""
    gen = torch.Generator(device="cuda").manual_seed(steps)
    g = O.matrix(70, 130, "noise", gen).to(O.TYPES[dtype])
    lift = 2.0 ** round(-steps * math.log2(abs(factor)))
    out = torch.empty(g.shape, dtype=O.TYPES[result], device="cuda")
    B.orthogonalise([g], out=[out], steps=steps, coefficients=(factor, 0.0, 0.0), scale=lift)
    want = g.double() / g.double().pow(2).sum((1, 2), keepdim=True).sqrt() * (factor ** steps * lift)
    own = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[result]
    each = 2.0 ** -12 if result == "bf16" else 2.0 ** -23
    # elements of 1 / 95 in the mean: of the bound on singular values, 1, two parts are rounded to 2^-39
    assert float((out.double() - want).norm() / want.norm()) < own + steps * (each + 2.0 ** -39 * 95)
    assert B.operator_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("steps,coefficients", [(12, (0.3, 0.2, 0.1)), (2, (0.0, 0.5, 0.25)), (6, [(0.1, 0.0, 0.0), (3.0, -3.5, 1.5)] * 3),
                                                (2, [(0.01, 0.02, 0.0), (60.0, -20.0, 3.0)]), (4, [(20.0, -19.5, 0.0), (0.05, 0.0, 0.0)] * 2)])
def test_values_that_shrink_and_grow(steps, coefficients, dtype):
    """Of an orthogonal matrix (singular values of 1 / 8) and of noise: what the operands of each step are rounded by, as for other
    polynomials.  Singular values lie 8 times below the bounds that the host derives, and 1000 times in the second step of (0, 0.5, 0.25)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    per = coefficients if isinstance(coefficients, list) else [coefficients] * steps
    orthogonal = torch.linalg.qr(torch.randn((2, 64, 64), generator=gen, device="cuda", dtype=torch.float64))[0].contiguous()
    for g in (orthogonal.to(O.TYPES[dtype]), O.matrix(96, 160, "noise", gen).to(O.TYPES[dtype])):
        want = O.exact(g, coefficients=per)
        lift = 2.0 ** -round(math.log2(float(want.abs().amax())))
        out = B.orthogonalise([g], out=[torch.empty_like(g)], steps=steps, coefficients=coefficients, scale=lift)[0]
        assert O.far(out, want * lift) < O.limit(dtype, steps=max(steps, 5))
    assert B.operator_status() == 0


@pytest.mark.parametrize("velocity", [False, True])
def test_what_is_carried_from_step_to_step_has_two_parts(velocity):
    """For 8-bit results too: 20 steps of a factor alone are off by 20 * 2^-23 at most.  Between two neighbouring results, 2^-8 to 2^-7 of them apart,
    1.2e-3 of all may then be rounded the other way than the exact value: sqrt(1.2e-3) * 2^-7.5 of the result's norm."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    g, v = O.matrix(200, 300, "noise", gen).bfloat16(), O.matrix(200, 300, "noise", gen)
    out = torch.empty_like(g)
    B.orthogonalise([g], out=[out], velocity=[v.clone()] if velocity else None, nesterov=False, momentum=0.5, steps=20, coefficients=(0.5, 0.0, 0.0),
                    scale=2.0 ** 20)
    u = g.double() + (0.5 * v.double() if velocity else 0.0)
    want = u / u.pow(2).sum((1, 2), keepdim=True).sqrt()
    assert O.far(out, want.bfloat16().double()) < 2.0 ** -12
