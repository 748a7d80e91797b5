"""The norm of attention heads with the rotation by position, and its gradients, against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
#: Half a unit in the last place of a result, relative (24, 8 and 11 significant bits), and half a step below fp16's normal range.
ROUND = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 0.0, "bf16": 0.0, "fp16": 2.0 ** -25}


def inputs(P, n, hq, hk, d, dtype, seed=0, spread=0):
    """(heads' inputs, gradients of the outputs, vectors); `spread` > 0: parts of wider rows."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    x = [(normal(P, n, h, d + spread) * 1.3).to(dt)[..., spread:] for h in (hq, hk)]
    g = [normal(P, n, h, d).to(dt) for h in (hq, hk)]
    w = [(1 + 0.1 * normal(P, d)).to(dt) for _ in range(2)]
    return x, g, w


def rotate(z, positions, rotary, base, interleaved):
    lead, rest = z[..., :rotary], z[..., rotary:]
    angle = positions.double()[:, :, None, None] * base ** (-torch.arange(0, rotary, 2, device="cuda").double() / max(1, rotary))
    cos, sin = torch.cos(angle), torch.sin(angle)
    a, b = (lead[..., 0::2], lead[..., 1::2]) if interleaved else (lead[..., :rotary // 2], lead[..., rotary // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def exact(x, w, positions, rotary, base, interleaved, eps):
    """(result, norm of x, z) in 64 bits."""
    v = x.double()
    xh = v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps) if w is not None else v
    z = xh * w.double()[:, None, None] if w is not None else xh
    return rotate(z, positions, rotary, base, interleaved), xh, z


def check(got, want, amplitude, dtype, operations, what):
    """A rounding of the result, and `operations` of 2^-24 of what it is put together from."""
    bound = ROUND[dtype] * 1.001 * want.abs() + 2.0 ** -24 * operations * amplitude + TINY[dtype]
    bad = (got.double() - want).abs() > bound
    assert not bad.any(), (what, int(bad.sum()), float(((got.double() - want).abs() / bound).max()))


def run_and_check(x, g, w, dtype, positions=None, rotary=None, base=10000.0, interleaved=False, eps=1e-6, backward=True):
    P, n, _, d = x[0].shape
    how = dict(w_q=w[0], w_k=w[1], positions=positions, rotary=rotary, base=base, interleaved=interleaved, eps=eps)
    at = torch.arange(n, device="cuda").expand(P, n) if positions is None else positions
    r = d // 2 * 2 if rotary is None else rotary
    outs = B.head_norm(*x, **how)
    if backward:
        *dxs, dws = B.head_norm_backward(*g, *x, **how)
    for m in range(2):
        if x[m] is None:
            assert outs[m] is None
            continue
        leaf, wl = x[m].double().requires_grad_(), None if w[m] is None else w[m].double().requires_grad_()
        want, xh, z = exact(leaf, wl, at, r, base, interleaved, eps)
        # sums of d squares along a tree, a root, a quotient, two products; sine and cosine within 2^-22; the turn's products
        ops = 24 + 4 * math.sqrt(d)
        size = lambda v: v.detach().abs().amax(-1, keepdim=True).expand_as(v)  # noqa: E731
        check(outs[m], want.detach(), 1.5 * size(z), dtype, ops, "qk"[m])
        if not backward:
            continue
        got = torch.autograd.grad(want, [leaf] + ([wl] if wl is not None else []), g[m].double())
        dz = rotate(g[m].double(), -at.double(), r, base, interleaved)
        inv = 1.0 if w[m] is None else 1 / torch.sqrt(leaf.detach().pow(2).mean(-1, keepdim=True) + eps)
        dzw = dz if w[m] is None else dz * w[m].double()[:, None, None]
        xh = xh.detach()
        parts = inv * (1.5 * size(dzw) + (size(xh) * (dzw * xh).abs().mean(-1, keepdim=True) if w[m] is not None else 0.0))
        check(dxs[m], got[0], parts, dtype, 2 * ops, "d" + "qk"[m])
        if w[m] is None:
            assert dws[m] is None
            continue
        terms = n * x[m].shape[2]
        # two sums of dz may fall on one element of 1.5 its size; sums along a fixed tree
        amplitude = 1.5 * (size(dz) * xh.abs()).sum((1, 2))
        check(dws[m], got[1], amplitude, dtype, ops + 4 * math.sqrt(terms), "dw_" + "qk"[m])


SIZES = [(1, 1, 1, 1, 64), (4, 1, 16, 4, 64), (2, 33, 3, 1, 128), (3, 200, 5, 5, 90), (2, 700, 8, 2, 96), (16, 9, 4, 4, 256), (1, 40, 2, 1, 80),
         (2, 65, 7, 7, 36), (1, 3, 1, 1, 2), (700, 2, 2, 1, 16)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("P,n,hq,hk,d", SIZES)
def test_sizes(P, n, hq, hk, d, interleaved, dtype):
    x, g, w = inputs(P, n, hq, hk, d, dtype)
    run_and_check(x, g, w, dtype, interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(64, 0), (64, 2), (64, 16), (64, 32), (64, 48), (64, 62), (90, 46), (127, 64), (1, 0), (255, 254), (3, 2),
                                      (248, 8), (8, 8), (24, 8), (24, 16), (65, 64), (256, 128)])
def test_parts_of_a_head(d, rotary, interleaved, dtype):
    x, g, w = inputs(2, 50, 3, 2, d, dtype, seed=1)
    run_and_check(x, g, w, dtype, rotary=rotary, interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 64])
def test_positions(bits, dtype):
    """Any size and sign, of any strides; the same for all replicas."""
    x, g, w = inputs(3, 40, 4, 2, 64, dtype, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for far in (10, 100000, 2 ** 31 - 1) + ((2 ** 45,) if bits == 64 else ()):
        p = torch.randint(-far, far, (3, 40), generator=gen, device="cuda")
        wide = torch.zeros((3, 90), dtype=torch.int32 if bits == 32 else torch.int64, device="cuda")
        at = wide[:, 4:84:2]
        at.copy_(p)
        # the oracle's own angle is within 2^-52 of a position times a frequency of at most 1: 2^-7 at 2^45, so only to 2^40
        if far <= 2 ** 31:
            run_and_check(x, g, w, dtype, positions=at)
            run_and_check(x, g, w, dtype, positions=at[:1].expand(3, 40), base=500000.0)
        else:
            q, k = B.head_norm(*x, w_q=w[0], w_k=w[1], positions=at)
            assert torch.isfinite(q).all() and torch.isfinite(k).all()


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
@pytest.mark.parametrize("given", [(True, False), (False, True), (False, False)])
def test_without_the_norm(given, dtype):
    x, g, w = inputs(2, 70, 4, 3, 64, dtype, seed=4)
    w = [v if on else None for v, on in zip(w, given)]
    run_and_check(x, g, w, dtype)
    run_and_check(x, g, w, dtype, rotary=0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_queries_alone(dtype):
    x, g, w = inputs(2, 70, 4, 3, 64, dtype, seed=5)
    run_and_check([x[0], None], [g[0], None], [w[0], None], dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("spread", [1, 8])
def test_parts_of_a_projection(spread, dtype):
    """Strided inputs off and on the 16-byte boundaries; results into parts of a buffer whose rest stays; results in place."""
    P, n, hq, hk, d = 2, 37, 4, 2, 64
    x, g, w = inputs(P, n, hq, hk, d, dtype, seed=6, spread=spread)
    run_and_check(x, g, w, dtype)
    dt = TYPES[dtype]
    buf = torch.full((P, n, hq + 2 * hk, d + spread), 7.0, dtype=dt, device="cuda")
    parts = buf[:, :, :hq, spread:], buf[:, :, hq:hq + hk, spread:]
    how = dict(w_q=w[0], w_k=w[1])
    want = B.head_norm(*x, **how)
    got = B.head_norm(*x, q_out=parts[0], k_out=parts[1], **how)
    assert got[0] is parts[0] and all(torch.equal(a, b) for a, b in zip(want, parts))
    dq, dk, dw = B.head_norm_backward(*g, *x, **how)
    d_w = torch.zeros((P, 3 * d), dtype=dt, device="cuda")
    r = B.head_norm_backward(*g, *x, dq=parts[0], dk=parts[1], d_weights=(d_w[:, :d], d_w[:, d + 3:2 * d + 3]), **how)
    assert r[0] is parts[0] and torch.equal(parts[0], dq) and torch.equal(parts[1], dk)
    assert torch.equal(d_w[:, :d], dw[0]) and torch.equal(d_w[:, d + 3:2 * d + 3], dw[1]) and (d_w[:, d:d + 3] == 0).all()
    assert (buf[:, :, hq + hk:] == 7.0).all() and (buf[..., :spread] == 7.0).all()
    # some of the results are not wanted
    _, _, (a, b) = B.head_norm_backward(*g, *x, d_weights=(None, d_w[:, :d]), **how)
    assert a is None and torch.equal(b, dw[1])
    # in place (copies are contiguous: other sums than those of the parts off the boundaries)
    mine = [v.clone() for v in x]
    want = B.head_norm(*mine, **how)
    B.head_norm(*mine, q_out=mine[0], k_out=mine[1], **how)
    assert all(torch.equal(a, b) for a, b in zip(mine, want))
    mine = [v.clone() for v in g]
    B.head_norm_backward(*mine, *x, dq=mine[0], dk=mine[1], **how)
    assert torch.equal(mine[0], dq) and torch.equal(mine[1], dk)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 66])
def test_heads_before_rows(d, dtype):
    """[P, heads, rows, width] in memory, as attention may want it."""
    x, g, w = inputs(2, 30, 4, 2, d, dtype, seed=7)
    x = [v.transpose(1, 2).contiguous().transpose(1, 2) for v in x]
    run_and_check(x, g, w, dtype)
    want = B.head_norm(*x, w_q=w[0], w_k=w[1])
    outs = [torch.empty_like(v) for v in x]
    assert outs[0].stride(2) > outs[0].stride(1)
    B.head_norm(*x, w_q=w[0], w_k=w[1], q_out=outs[0], k_out=outs[1])
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_without_an_epsilon(dtype):
    x, g, w = inputs(3, 41, 5, 2, 64, dtype, seed=8)
    run_and_check(x, g, w, dtype, eps=0.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_row_that_is_not_finite_keeps_to_itself(bad):
    x, g, w = inputs(2, 41, 5, 2, 64, "fp32", seed=9)
    how = dict(w_q=w[0], w_k=w[1])
    q, _ = B.head_norm(*x, **how)
    dq, dk, dw = B.head_norm_backward(*g, *x, **how)
    x[0][1, 7, 3, 5] = bad
    q2, _ = B.head_norm(*x, **how)
    dq2, dk2, dw2 = B.head_norm_backward(*g, *x, **how)
    rest = torch.ones(2, 41, 5, dtype=torch.bool, device="cuda")
    rest[1, 7, 3] = False
    assert torch.equal(q[rest], q2[rest]) and torch.equal(dq[rest], dq2[rest]) and torch.equal(dk, dk2)
    assert not torch.isfinite(q2[1, 7, 3]).all()
    assert torch.equal(dw[1], dw2[1]) and torch.equal(dw[0][0], dw2[0][0])


def test_no_rows():
    x, g, w = inputs(2, 0, 3, 1, 64, "bf16")
    q, k = B.head_norm(*x, w_q=w[0], w_k=w[1])
    assert q.shape == (2, 0, 3, 64) and k.shape == (2, 0, 1, 64)
    dq, dk, dw = B.head_norm_backward(*g, *x, w_q=w[0], w_k=w[1])
    assert dq.shape == q.shape and (dw[0] == 0).all() and (dw[1] == 0).all()


def test_gradients_against_differences():
    """Central differences of the forward pass along random directions; widths that 32 bits still resolve."""
    x, g, w = inputs(1, 12, 2, 1, 32, "fp32", seed=10)
    how = dict(rotary=20)
    loss = lambda q, k, wq, wk: sum((o.double() * d.double()).sum() for o, d in zip(B.head_norm(q, k, w_q=wq, w_k=wk, **how), g))  # noqa: E731
    dq, dk, dw = B.head_norm_backward(*g, *x, w_q=w[0], w_k=w[1], **how)
    h = 2.0 ** -7
    for seed in range(3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        v = [torch.randn(t.shape, generator=gen, device="cuda") for t in (*x, *w)]
        step = lambda s: [t + s * h * u for t, u in zip((*x, *w), v)]  # noqa: E731
        slope = (loss(*step(1)) - loss(*step(-1))) / (2 * h)
        by_hand = sum((t.double() * u.double()).sum() for t, u in zip((dq, dk, *dw), v))
        size = sum((t.double() * u.double()).pow(2).sum() for t, u in zip((dq, dk, *dw), v)).sqrt()
        # third derivatives times h^2 / 6 (some ten times 1e-5) and roundings of 2^-24 / h: below 1 % of the summands' size
        assert abs(slope - by_hand) < 1e-2 * size, (float(slope), float(by_hand), float(size))


def test_captured_and_replayed():
    x, g, w = inputs(2, 90, 4, 2, 64, "bf16", seed=11)
    at = torch.arange(90, device="cuda").repeat(2, 1)
    dq, dk = (torch.empty_like(v) for v in x)
    outs = [torch.empty_like(v) for v in x]
    d_w = [torch.empty_like(v) for v in w]

    def both():
        B.head_norm(*x, w_q=w[0], w_k=w[1], positions=at, q_out=outs[0], k_out=outs[1])
        B.head_norm_backward(*g, *x, w_q=w[0], w_k=w[1], positions=at, dq=dq, dk=dk, d_weights=d_w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (12, 13):
        x2, g2, w2 = inputs(2, 90, 4, 2, 64, "bf16", seed=seed)
        for to, v in zip((*x, *g, *w), (*x2, *g2, *w2)):
            to.copy_(v)
        at.add_(1000)
        graph.replay()
        want = B.head_norm(*x, w_q=w[0], w_k=w[1], positions=at)
        want_dq, want_dk, want_w = B.head_norm_backward(*g, *x, w_q=w[0], w_k=w[1], positions=at)
        for a, b in zip((*outs, dq, dk, *d_w), (*want, want_dq, want_dk, *want_w)):
            assert torch.equal(a, b)
    run_and_check(x, g, w, "bf16", positions=at)


def test_two_streams_at_once():
    sets = [inputs(2, 500, 8, 2, 128, "bf16", seed=s) for s in (14, 15)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = [[], []]
    for _ in range(10):
        for s, (x, g, w), out in zip(streams, sets, results):
            out.append(B.head_norm_backward(*g, *x, w_q=w[0], w_k=w[1], stream=s))
    torch.cuda.synchronize()
    for (x, g, w), out in zip(sets, results):
        run_and_check(x, g, w, "bf16")
        for r in out[1:]:
            assert torch.equal(r[0], out[0][0]) and torch.equal(r[1], out[0][1]) and all(torch.equal(a, b) for a, b in zip(r[2], out[0][2]))


def test_refusals():
    x, g, w = inputs(2, 10, 4, 2, 64, "fp32")
    q, k = x
    ok = dict(w_q=w[0], w_k=w[1])
    at = torch.zeros((2, 10), dtype=torch.int64, device="cuda")
    wide = torch.zeros((2, 10, 1, 258), device="cuda")
    calls = [lambda: B.head_norm(q[0], k, **ok), lambda: B.head_norm(q, k[0], **ok), lambda: B.head_norm(q, k.bfloat16(), **ok),
             lambda: B.head_norm(q.double(), k.double()), lambda: B.head_norm(q, k[:1], **ok), lambda: B.head_norm(q, k, w_q=w[0][:, :8]),
             lambda: B.head_norm(q, k, rotary=3, **ok), lambda: B.head_norm(q, k, rotary=66, **ok), lambda: B.head_norm(q, k, rotary=-2, **ok),
             lambda: B.head_norm(q, k, eps=-1.0, **ok), lambda: B.head_norm(q, k, eps=float("nan"), **ok), lambda: B.head_norm(q, k, base=0.0, **ok),
             lambda: B.head_norm(q, k, base=float("inf"), **ok), lambda: B.head_norm(q, k, positions=at.float(), **ok),
             lambda: B.head_norm(q, k, positions=at[:1], **ok), lambda: B.head_norm(q, k, positions=at.cpu(), **ok),
             lambda: B.head_norm(wide, None), lambda: B.head_norm(q, None, **ok), lambda: B.head_norm(q, None, k_out=k),
             lambda: B.head_norm(q.transpose(2, 3), k), lambda: B.head_norm(q, k, q_out=q[:, :1].expand(2, 10, 4, 64), **ok),
             lambda: B.head_norm(q[:, :, :1], k, q_out=q.as_strided((2, 10, 1, 64), (32, 64, 64, 1))),
             lambda: B.head_norm_backward(g[0], None, q, k, **ok), lambda: B.head_norm_backward(None, g[1], q, k, **ok),
             lambda: B.head_norm_backward(g[0], g[1], q, k, d_weights=(w[0], w[1])), lambda: B.head_norm_backward(*g, q, k, d_weights=(None,), **ok),
             lambda: B.head_norm_backward(*g, q, k, dq=q[:1].expand(2, 10, 4, 64), **ok), lambda: B.head_norm(q.cpu(), k.cpu())]
    for number, call in enumerate(calls):
        with pytest.raises(B.EventGradError):
            call()
            pytest.fail(str(number))
    with pytest.raises(B.EventGradError, match="no_grad"):
        B.head_norm(q.clone().requires_grad_(), k)
