"""The norm of attention heads and the rotation by position at the ends of their ranges."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

import test_gpu_head_norm as H
from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TURN = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def angles(positions, rotary, base):
    """Angles in radians, ``[places, rotary / 2]``, reduced to a turn in 60 digits before they become numbers of 64 bits."""
    getcontext().prec = 60
    turns = [(Decimal(base).ln() * (Decimal(-2 * j) / Decimal(rotary))).exp() / TURN for j in range(rotary // 2)]
    return torch.tensor([[float((Decimal(p) * t % 1) * TURN) for t in turns] for p in positions], dtype=torch.float64, device="cuda")


def test_the_oracle():
    near = angles([0, 1, -3, 1000], 8, 10000)
    want = torch.tensor([0.0, 1.0, -3.0, 1000.0], dtype=torch.float64, device="cuda")[:, None] * 10.0 ** -torch.arange(4, device="cuda").double()
    # Python's remainder has the sign of the first number: the same angle
    assert ((near - want).cos() - 1).abs().max() < 1e-12


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary,base", [(64, 64, 10000.0), (128, 128, 500000.0), (90, 46, 10000.0), (256, 256, 1e30), (36, 6, 1.0), (16, 16, 3.0)])
def test_far_positions(d, rotary, base, interleaved):
    """A frequency is below 2^61.4 units of 2^-64 of a turn.  It is a product of three exponentials (a unit in the last of 64 places each, with
    their arguments) and rounds three times on the way (half of one): 4.5 * 2^-64 of it, 0.75 units, and half a unit in the end."""
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 36 + 12345, -2 ** 40 + 77, 2 ** 40 + 1, 2 ** 45 - 3, -2 ** 45 - 12345678901]
    (q, _), _, (w, _) = H.inputs(1, len(positions), 3, 1, d, "fp32", seed=1)
    at = torch.tensor([positions], device="cuda")
    out, _ = B.head_norm(q, None, w_q=w, positions=at, rotary=rotary, base=base, interleaved=interleaved)
    x = q.double()
    z = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * w.double()[:, None, None]
    a = angles(positions, rotary, base)[None, :, None]
    lead = z[..., :rotary]
    u, v = (lead[..., 0::2], lead[..., 1::2]) if interleaved else (lead[..., :rotary // 2], lead[..., rotary // 2:])
    u, v = u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()
    want = torch.cat([torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1), z[..., rotary:]], -1)
    size = z.abs().amax(-1, keepdim=True)
    off = torch.tensor(positions, device="cuda").double().abs()[None, :, None, None] * 1.25 * 2.0 ** -64 * 2 * math.pi
    # a turned pair moves by the angle's error; the rest as in the tests of ordinary positions
    bound = 2.0 ** -24 * 1.001 * want.abs() + 1.5 * size * (2.0 ** -24 * (24 + 4 * math.sqrt(d)) + off)
    bad = (out.double() - want).abs() > bound
    assert not bad.any(), (bad.nonzero()[:5].tolist(), float(((out.double() - want).abs() / bound).max()))


def far_rows(dtype, sizes):
    """Heads of ordinary size, one of each kind multiplied by each of the sizes; which ones."""
    x, g, w = H.inputs(2, 37, 5, 2, 64, dtype, seed=12)
    plain = [t.clone() for t in x]
    for t in x:
        for k, size in enumerate(sizes):
            t[1, 3 * k + 1, k % t.shape[2]] *= size
    return x, plain, g, w, [(a != b).any(-1) for a, b in zip(x, plain)]


@pytest.mark.parametrize("d", [64, 67])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_whose_squares_pass_the_range(dtype, d):
    """As the header has it: their results are zeros, and the gradients with them; the other rows keep their bits."""
    x, plain, g, w, far = far_rows(dtype, [2.0 ** 68, 2.0 ** 100, 2.0 ** 118])
    if d == 67:                                          # off the 16-byte boundaries
        apart = [torch.zeros((*t.shape[:3], d), dtype=t.dtype, device="cuda")[..., 3:] for t in (*x, *plain)]
        for to, t in zip(apart, (*x, *plain)):
            to.copy_(t)
        x, plain = apart[:2], apart[2:]
    how = dict(w_q=w[0], w_k=w[1])
    for results in (lambda v: B.head_norm(*v, **how), lambda v: B.head_norm_backward(*g, *v, **how)[:2]):
        for rows, a, b in zip(far, results(x), results(plain)):
            assert int(rows.sum()) == 3 and (a[rows] == 0).all() and torch.equal(a[~rows], b[~rows])
    dws = [B.head_norm_backward(*g, *v, **how)[2] for v in (x, plain)]
    for a, b in zip(*dws):
        assert torch.isfinite(a).all() and torch.equal(a[0], b[0])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_whose_squares_sink_below_the_range(dtype):
    """Beside an epsilon they are what the formula makes them; without one they spoil nobody else's results."""
    x, plain, g, w, far = far_rows(dtype, [2.0 ** -40, 2.0 ** -70, 2.0 ** -100])
    H.run_and_check(x, g, w, dtype)
    x[0][0, 2, 1] = 0
    q, k = B.head_norm(*x, w_q=w[0], w_k=w[1])
    assert (q[0, 2, 1] == 0).all()
    far[0][0, 2, 1] = True
    how = dict(w_q=w[0], w_k=w[1], eps=0.0)
    for rows, a, b in zip(far, B.head_norm(*x, **how), B.head_norm(*plain, **how)):
        assert torch.equal(a[~rows], b[~rows]) and torch.isfinite(a[~rows]).all()
    assert torch.isnan(B.head_norm(*x, **how)[0][0, 2, 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shift,d", [(0, 63), (1, 62), (1, 63), (3, 9)])
def test_what_stands_beside_a_head_is_not_used(shift, d, dtype):
    """Single 16-bit values come as words of 4 bytes: NaN in the halves that belong to nobody, and heads that others write meanwhile, change nothing."""
    x, g, w = H.inputs(2, 41, 5, 2, d, dtype, seed=14)
    wide = [torch.full((*t.shape[:3], d + 5), float("nan"), dtype=t.dtype, device="cuda") for t in (*x, *g)]
    parts = [b[..., shift:shift + d] for b in wide]
    for to, t in zip(parts, (*x, *g)):
        to.copy_(t)
    H.run_and_check(parts[:2], parts[2:], w, dtype)
    how = dict(w_q=w[0], w_k=w[1])
    want = B.head_norm(*parts[:2], **how)
    # results into the same words: the inputs' neighbours change while they are read
    B.head_norm(*parts[:2], q_out=parts[0], k_out=parts[1], **how)
    assert all(torch.equal(a, b) for a, b in zip(parts, want))
    for b, p in zip(wide, parts):
        p.fill_(float("nan"))
        assert torch.isnan(b).all()
