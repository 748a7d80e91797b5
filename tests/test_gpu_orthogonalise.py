"""Orthogonal updates against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
DEFAULT = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)                  # converges


def matrix(rows, columns, kind, gen, P=2):
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    if kind == "noise":
        return normal(P, rows, columns)
    if kind == "rank":                    # one direction alone
        return normal(P, rows, 1) @ normal(P, 1, columns)
    k = min(rows, columns, 12)            # some directions of falling weight, over a little noise
    return (normal(P, rows, k) * torch.logspace(0, -2, k, device="cuda")) @ normal(P, k, columns) + 0.02 * normal(P, rows, columns)


def exact(u, steps=5, coefficients=None):
    x = u.double()
    flip = x.shape[1] > x.shape[2]
    x = x if not flip else x.mT
    x = x / x.pow(2).sum((1, 2), keepdim=True).sqrt()
    x = x.mT                              # rows >= columns above, wide from here on
    per = coefficients or [DEFAULT] * steps
    for a, b, c in per:
        gram = x @ x.mT
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x if flip else x.mT


def far(got, want):
    return float((got.double() - want).norm() / want.norm())


def limit(dtype, steps=5, few=False):
    """Of |error| / |result|, in the Frobenius norm.

    A product is off by what its operands were rounded by (22 bits: 2^-22 / sqrt(3) in the mean with what is left out; 11 bits:
    2^-11 / sqrt(3) of both) and, in full precision, by the accumulator's truncation: 2^-25 for each of the 16 additions between two
    hand-overs to registers, all towards zero.  With x a square of a singular value, an error d of all three products of a step
    changes its result by up to d (|b| x + 3 c x^2 + |b x + c x^2|): 10 d at x = 0.8, where the values settle.  The truncations of five steps
    may add up; roundings have random signs: sqrt(10) instead of 10, sqrt(steps) instead of steps, times 2 for the slope of the
    polynomial between steps (1.1 at most from 0.7 to 1, 3.9 at its very end).

    `few`: the weight lies in few directions, and what roundings leave in the others grows 3.4445 times a step.  The gradient's own
    (2^-24 of an element) grows 484 times.  Two steps in one add 11.9 X (a0 a1) and a product that takes most of it away where the weight is: three
    roundings of 2^-24 of 11.9 of an element, sqrt(3) * 11.9, which grow 41 times after the first two steps and 3.4 times after the
    next two.  (Results of 8 bits carry X through the steps in 22 bits: below their own rounding.)"""
    if dtype == "bf16":
        return 2 * math.sqrt(10 * steps) * 2.0 ** -11 / math.sqrt(3) + 2.0 ** -9
    own = {"fp32": 2.0 ** -25, "fp16": 2.0 ** -12}[dtype]
    return steps * 10 * 16 * 2.0 ** -25 + 2 * math.sqrt(10 * steps) * 2.0 ** -22 / math.sqrt(3) + ((484 + math.sqrt(3) * 11.9 * (41 + 3.4)) * 2.0 ** -24 if few else 0.0) + own


SIZES = [(1, 1), (1, 7), (10, 32), (64, 64), (64, 784), (65, 63), (27, 64), (128, 128), (129, 257), (300, 200), (256, 576), (520, 515), (1000, 70), (3, 5000),
         (1024, 700), (768, 1100)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,columns", SIZES)
@pytest.mark.parametrize("kind", ["noise", "fall", "rank"])
def test_sizes(rows, columns, kind, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + columns)
    g = (matrix(rows, columns, kind, gen) * 1e-3).to(TYPES[dtype])
    out = torch.full_like(g, 9.0)
    r = B.orthogonalise([g], out=[out])
    assert r[0] is out
    want = exact(g)
    assert B.operator_status() == 0
    print(far(out, want) / limit(dtype, few=kind != "noise"))
    assert far(out, want) < limit(dtype, few=kind != "noise")
    again = torch.empty_like(out)
    B.orthogonalise([g], out=[again])
    assert torch.equal(out, again)


def make(shapes, dtype, P=2, seed=0, velocity=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    grads = [matrix(r, c, "fall", gen, P).to(TYPES[dtype]) for r, c in shapes]
    return grads, [matrix(r, c, "fall", gen, P) for r, c in shapes] if velocity else None


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("dtype,result", [("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32")])
def test_many_matrices_with_momentum(dtype, result, nesterov):
    """Of different sizes and sides in one call; some without a velocity."""
    shapes = [(64, 784), (32, 64), (10, 32), (300, 100), (513, 260), (1, 40), (128, 640)]
    grads, velocity = make(shapes, dtype)
    before = [v.clone() for v in velocity]
    given = [None if k == 2 else v for k, v in enumerate(velocity)]
    out = [torch.full(g.shape, 9.0, dtype=TYPES[result], device="cuda") for g in grads]
    B.orthogonalise(grads, out=out, velocity=given, momentum=0.9, nesterov=nesterov)
    for k, (g, v, v0, o) in enumerate(zip(grads, velocity, before, out)):
        u = g.double()
        if k != 2:
            v1 = 0.9 * v0.double() + u
            # momentum in 32 bits (2^-24 of it), a product and a sum that round once
            assert ((v.double() - v1).abs() <= 2.0 ** -24 * 1.001 * (v1.abs() + (0.9 * v0.double()).abs())).all()
            u = u + 0.9 * v1 if nesterov else v1
        assert far(o, exact(u)) < limit(result, few=True), k
    assert torch.equal(velocity[2], before[2])
    # the velocity somewhere else: the same, and the old one stays
    fresh, out2 = [torch.empty_like(v) for v in velocity], [torch.empty_like(o) for o in out]
    old = [v.clone() for v in before]
    B.orthogonalise(grads, out=out2, velocity=old, velocity_out=fresh, momentum=0.9, nesterov=nesterov)
    for k in range(len(shapes)):
        assert torch.equal(old[k], before[k])
        if k != 2:
            assert torch.equal(fresh[k], velocity[k]) and torch.equal(out2[k], out[k])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_in_place_and_scaled(dtype):
    grads, _ = make([(70, 200), (200, 70)], dtype, velocity=False)
    want = [g.clone() for g in grads]
    out = [torch.empty_like(g) for g in grads]
    B.orthogonalise(want, out=out, scale=[0.5, -2.0])
    given = tuple(grads)
    r = B.orthogonalise(given, scale=[0.5, -2.0])
    assert r[0] is grads[0] and all(torch.equal(a, b) for a, b in zip(grads, out))
    for o, w, s in zip(out, want, (0.5, -2.0)):
        assert far(o, s * exact(w)) < limit(dtype, few=True)


@pytest.mark.parametrize("dtype,result", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("rows,columns", [(70, 201), (201, 70), (64, 128), (33, 33)])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_views_of_any_stride(shift, rows, columns, dtype, result):
    """Parts of larger buffers, replicas one after the other or in turn; nothing else of the buffers changes."""
    P = 3
    gen = torch.Generator(device="cuda").manual_seed(5)
    g, v = matrix(rows, columns, "fall", gen, P).to(TYPES[dtype]), matrix(rows, columns, "fall", gen, P)

    def apart(dt):
        whole = torch.full((P, rows + 2, columns + 9), 7.0, dtype=dt, device="cuda")
        return whole, whole[:, 1:rows + 1, shift:shift + columns]

    def in_turn(dt):
        whole = torch.full((rows, P, columns + 9), 7.0, dtype=dt, device="cuda")
        return whole, whole[:, :, shift:shift + columns].transpose(0, 1)
    want, want_v = torch.empty(g.shape, dtype=TYPES[result], device="cuda"), torch.empty_like(v)
    B.orthogonalise([g], out=[want], velocity=[v], velocity_out=[want_v])
    u = g.double() + 0.95 * (0.95 * v.double() + g.double())
    assert far(want, exact(u)) < limit(result, few=True)
    for form in (apart, in_turn):
        (_, gs), (vb, vs), (ob, os_) = form(TYPES[dtype]), form(torch.float32), form(TYPES[result])
        gs.copy_(g), vs.copy_(v)
        B.orthogonalise([gs], out=[os_], velocity=[vs])
        # the order of the sum of squares follows the layout: the norm may differ in its last place
        assert far(os_, want.double()) < 2 * limit(result, few=True)
        assert torch.equal(vs, want_v)
        for whole, part in ((vb, vs), (ob, os_)):
            part.fill_(7.0)
            assert (whole == 7.0).all()
    # one gradient for all replicas is read, never written
    same = g[:1].expand(P, rows, columns)
    o = torch.empty(g.shape, dtype=TYPES[result], device="cuda")
    B.orthogonalise([same], out=[o])
    assert torch.equal(o[0], o[1]) and far(o, exact(same.double())) < limit(result, few=True)
    with pytest.raises(B.EventGradError):
        B.orthogonalise([same])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_zeros_and_values_that_are_not_finite(dtype):
    """A matrix of zeros gives zeros, one with an infinity or NaN gives NaN, each in its own replica and matrix."""
    grads, _ = make([(60, 100), (200, 130)], dtype, P=4, velocity=False)
    clean = [torch.empty_like(g) for g in grads]
    B.orthogonalise(grads, out=clean)
    grads[0][1] = 0
    grads[0][2, 5, 7] = float("nan")
    grads[1][3, 5, 7] = float("inf")
    out = [torch.full_like(g, 9.0) for g in grads]
    B.orthogonalise(grads, out=out)
    assert (out[0][1] == 0).all() and torch.isnan(out[0][2]).all() and torch.isnan(out[1][3]).all()
    assert torch.equal(out[0][[0, 3]], clean[0][[0, 3]]) and torch.equal(out[1][:3], clean[1][:3])


@pytest.mark.parametrize("dtype,sizes", [("fp32", (1e-38, 1e-30, 1e-6, 1e6, 1e18, 1e36)), ("bf16", (1e-38, 1e-30, 1e6, 1e36)), ("fp16", (1e-4, 1.0, 1e4))])
def test_gradients_of_any_size(dtype, sizes):
    """Scaled by a power of two a gradient has the same bits in its result, far beyond where squares pass 32 bits."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    for size in sizes:
        g = (matrix(70, 90, "noise", gen) * size).to(TYPES[dtype])
        out = B.orthogonalise([g], out=[torch.empty_like(g)])[0]
        assert far(out, exact(g)) < limit(dtype)
        if size in (1e-6, 1.0, 1e6):
            # (upwards: a quarter of fp16's smallest values would be rounded)
            again = B.orthogonalise([g * 4.0], out=[torch.empty_like(g)])[0]
            assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("steps,coefficients", [(1, None), (2, None), (8, None), (6, CUBIC), (10, (1.875, -1.25, 0.375)),
                                                (3, [(4.0, -6.0, 2.9), (3.0, -3.5, 1.5), (1.875, -1.25, 0.375)]), (2, (0.0, 1.0, 0.0)), (1, (8.0, 2.0, 1.0))])
def test_steps_and_coefficients(steps, coefficients, dtype):
    gen = torch.Generator(device="cuda").manual_seed(9)
    g = matrix(130, 200, "noise", gen).to(TYPES[dtype])
    per = coefficients if isinstance(coefficients, list) else [coefficients or DEFAULT] * steps
    out = B.orthogonalise([g], out=[torch.empty_like(g)], steps=steps, coefficients=coefficients)[0]
    assert far(out, exact(g, coefficients=per)) < limit(dtype, steps=max(steps, 5))
    if steps == 10:                                    # converged
        assert float((out.double() @ out.double().mT - torch.eye(130, device="cuda")).abs().max()) < (1e-4 if dtype == "fp32" else 0.05)


@pytest.mark.parametrize("kind,dtype,steps,coefficients", [
    ("noise", "fp32", 5, None), ("fall", "fp32", 5, None), ("rank", "fp32", 5, None), ("noise", "fp16", 5, None), ("rank", "fp16", 5, None),
    ("noise", "fp32", 2, None), ("noise", "fp32", 8, None), ("noise", "fp32", 6, CUBIC),
    ("noise", "fp32", 3, [(4.0, -6.0, 2.9), (3.0, -3.5, 1.5), (1.875, -1.25, 0.375)]), ("noise", "fp32", 2, [(0.5, 1.0, 0.0), (3.0, -3.5, 1.5)])])
def test_two_steps_in_one(kind, dtype, steps, coefficients):
    """Of wide matrices with work for it, small ones among them: P m^2 (n - 2 m) is 2.3e9."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    grads = [matrix(*size, kind, gen).to(TYPES[dtype]) for size in ((640, 4100), (33, 70), (300, 129))]
    per = coefficients if isinstance(coefficients, list) else [coefficients or DEFAULT] * steps
    for g, o in zip(grads, B.orthogonalise(grads, out=[torch.empty_like(g) for g in grads], steps=steps, coefficients=coefficients)):
        assert far(o, exact(g, coefficients=per)) < limit(dtype, steps=max(steps, 5), few=kind != "noise")
    assert B.operator_status() == 0


@pytest.mark.parametrize("rows,columns", [(3, 2 ** 18), (2 ** 18 + 65, 2), (1, 2 ** 20)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_sides(rows, columns, dtype):
    """Sums over up to 2^20 values.  In full precision a hand-over every 4 steps keeps the limit that of any length.  A sum of 8-bit
    results (up to 2^18) stays in the accumulator: each of its n / 16 additions truncates up to 2^-23 of it, which makes A less by up to
    n / 16 * 2^-23 in every step, times 10 for what a step makes of it (see limit), 5 steps."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((1, min(rows, columns), max(rows, columns)), generator=gen, device="cuda").to(TYPES[dtype])
    g = x if rows <= columns else x.mT.contiguous()
    out = B.orthogonalise([g], out=[torch.empty_like(g)])[0]
    want = x.double()
    want = want / want.norm()
    for _ in range(5):
        gram = want @ want.mT
        want = DEFAULT[0] * want + (DEFAULT[1] * gram + DEFAULT[2] * gram @ gram) @ want
    n = max(rows, columns)
    bound = limit(dtype) + (n / 16 * 2.0 ** -23 * 10 * 5 if dtype == "bf16" and n <= 2 ** 18 else 0.0)
    assert far(out if rows <= columns else out.mT, want) < bound
    assert B.operator_status() == 0


def test_matrices_that_share_no_launches():
    """More than one group: by number, and by memory."""
    grads, _ = make([(16, 24)] * 100, "bf16", P=1, velocity=False)
    out = B.orthogonalise(grads, out=[torch.empty_like(g) for g in grads])
    for g, o in list(zip(grads, out))[::9]:
        assert far(o, exact(g)) < limit("bf16", few=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    big = [matrix(1024, 4096, "noise", gen, P=4).bfloat16() for _ in range(7)]
    out = B.orthogonalise(big, out=[torch.empty_like(g) for g in big])
    for g, o in zip(big, out):
        assert far(o, exact(g)) < limit("bf16")
    assert B.operator_status() == 0


def test_captured_and_replayed_with_other_gradients():
    grads, velocity = make([(64, 200), (300, 90)], "bf16")
    out = [torch.empty(g.shape, device="cuda") for g in grads]

    def call():
        B.orthogonalise(grads, out=out, velocity=velocity)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (4, 5):
        g2, v2 = make([(64, 200), (300, 90)], "bf16", seed=seed)
        for to, v in zip((*grads, *velocity), (*g2, *v2)):
            to.copy_(v)
        graph.replay()
        want = [torch.empty_like(o) for o in out]
        B.orthogonalise(g2, out=want, velocity=v2)
        assert all(torch.equal(a, b) for a, b in zip((*out, *velocity), (*want, *v2)))


def test_two_streams_at_once():
    sets = [make([(300, 500), (64, 64)], "fp32", seed=s, velocity=False)[0] for s in (6, 7)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = [[], []]
    for _ in range(6):
        for s, grads, kept in zip(streams, sets, results):
            with torch.cuda.stream(s):
                out = [torch.empty_like(g) for g in grads]
            kept.append(B.orthogonalise(grads, out=out, stream=s))
    torch.cuda.synchronize()
    for grads, kept in zip(sets, results):
        for g, o in zip(grads, kept[0]):
            assert far(o, exact(g)) < limit("fp32", few=True)
        assert all(torch.equal(a, b) for r in kept[1:] for a, b in zip(r, kept[0]))


def test_into_the_buffer_of_the_step():
    """Gradients in bf16 become fp32 updates in the buffer that clipping and the step read; vectors between them stay."""
    P, shapes = 3, [(40, 72), (72,), (10, 40), (130, 70)]
    ring = B.EventGrad(P, [math.prod(s) for s in shapes])
    gen = torch.Generator(device="cuda").manual_seed(1)
    grads = torch.randn((P, ring.replica_stride), generator=gen, device="cuda").bfloat16()
    updates = ring.empty_params()
    updates.fill_(3.0)
    at = [t for t, s in enumerate(shapes) if len(s) == 2]
    views = lambda buf: [ring.view(buf, t, shapes[t]) for t in at]  # noqa: E731
    B.orthogonalise(views(grads), out=views(updates), scale=[0.2 * max(shapes[t]) ** 0.5 for t in at])
    for t, o, g in zip(at, views(updates), views(grads)):
        assert far(o, 0.2 * max(shapes[t]) ** 0.5 * exact(g)) < limit("fp32")
    assert (ring.view(updates, 1, (72,)) == 3.0).all()
    params = ring.empty_params()
    params.zero_()
    ring.clip_gradients(updates, 1e6)
    before = updates.clone()
    ring.step(params, updates, 0.1)
    for t in at:
        assert torch.equal(ring.view(params, t, shapes[t]), -0.1 * ring.view(before, t, shapes[t]))
    ring.close()


def test_refusals():
    g = torch.randn((2, 8, 12), device="cuda")
    h = g.bfloat16()
    calls = [lambda: B.orthogonalise([g[0]]), lambda: B.orthogonalise([g, g[:1].clone()]), lambda: B.orthogonalise([g, h]), lambda: B.orthogonalise([g.double()]),
             lambda: B.orthogonalise([g.int()]), lambda: B.orthogonalise([g.cpu()]), lambda: B.orthogonalise([g.transpose(1, 2)]), lambda: B.orthogonalise([g, g]),
             lambda: B.orthogonalise([g], out=[h]), lambda: B.orthogonalise([h], out=[h.half()]), lambda: B.orthogonalise([g], out=[]),
             lambda: B.orthogonalise([g], out=[g[:, :4]]), lambda: B.orthogonalise([g], velocity=[h]), lambda: B.orthogonalise([g], velocity=[g]),
             lambda: B.orthogonalise([g], velocity_out=[torch.empty_like(g)]), lambda: B.orthogonalise([g], velocity=[g.clone(), None]),
             lambda: B.orthogonalise([g], steps=0), lambda: B.orthogonalise([g], steps=65), lambda: B.orthogonalise([g], coefficients=(1.0, 2.0)),
             lambda: B.orthogonalise([g], coefficients=[(1.0, 0.0, 0.0)] * 4), lambda: B.orthogonalise([g], coefficients=(5.0, 0.0, 0.0)),
             lambda: B.orthogonalise([g], scale=[1.0, 2.0]), lambda: B.orthogonalise([g], scale=float("nan")), lambda: B.orthogonalise([g], momentum=float("nan"), velocity=[g.clone()]),
             lambda: B.orthogonalise([g], out=[g[:, :1].expand(2, 8, 12)]), lambda: B.orthogonalise([g[:, :0]]), lambda: B.orthogonalise([None])]
    for number, call in enumerate(calls):
        with pytest.raises(B.EventGradError):
            call()
            pytest.fail(str(number))
    with pytest.raises(B.EventGradError, match="no_grad"):
        B.orthogonalise([g.clone().requires_grad_()])
    assert B.orthogonalise([]) == ()
