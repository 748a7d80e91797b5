"""The norm between two residual blocks and its gradients against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
#: Half a unit in the last place of a result, relative (24, 8 and 11 significant bits).
ROUND = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
NAMES = ("w_post", "gate", "scale", "w_pre")


def inputs(P, n, d, dtype, seed=0, given=NAMES, spread=0):
    """Random inputs; `spread` > 0 makes the rows `d + spread` apart."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]

    def rows(scale):
        t = torch.randn((P, n, d + spread), generator=gen, device="cuda") * scale
        return t.to(dt)[:, :, :d]

    def vec(mean, dev):
        t = mean + dev * torch.randn((P, d + 3 * spread), generator=gen, device="cuda")
        return t.to(dt)[:, :d]

    x = dict(y=rows(0.7), residual=rows(1.3), d_r=rows(0.1), d_o=rows(0.1))
    w = dict(w_post=vec(1, 0.1), gate=vec(0, 1.0), scale=vec(1, 0.1), w_pre=vec(1, 0.1))
    return x, {k: (v if k in given else None) for k, v in w.items()}


def exact(x, w, eps, use=("d_r", "d_o")):
    """Forward and gradients in 64 bits, the latter by differentiating the former."""
    leaf = {k: v.double().requires_grad_() for k, v in list(x.items())[:2] if v is not None}
    wl = {k: v.double().requires_grad_() for k, v in w.items() if v is not None}
    rms = lambda v: v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps)  # noqa: E731
    r = leaf["residual"]
    if "scale" in wl:
        r = wl["scale"][:, None] * r
    if "y" in leaf:
        u = leaf["y"]
        if "w_post" in wl:
            u = rms(u) * wl["w_post"][:, None]
        if "gate" in wl:
            u = torch.sigmoid(wl["gate"])[:, None] * u
        r = r + u
    o = rms(r) * wl["w_pre"][:, None] if "w_pre" in wl else None
    total = 0.0
    if "d_r" in use:
        total = total + (r * x["d_r"].double()).sum()
    if "d_o" in use and o is not None:
        total = total + (o * x["d_o"].double()).sum()
    names = list(leaf) + list(wl)
    grads = dict(zip(names, torch.autograd.grad(total, [*leaf.values(), *wl.values()], allow_unused=True)))
    return r.detach(), None if o is None else o.detach(), grads


def amplitudes(x, w, eps, use):
    """Sizes of the summands of dr and dy, which cancel in part (wholly for a width of one): row maxima of
    scale * (|d_r| + inv2 (|dn| + |rh c3|)) and of inv1 * a * (that) * (1 + |yh|)."""
    col = {k: (1.0 if v is None else v.double()[:, None]) for k, v in w.items()}
    y, r = (0.0 if x[k] is None else x[k].double() for k in ("y", "residual"))
    inv1 = torch.rsqrt(y.pow(2).mean(-1, keepdim=True) + eps) if w["w_post"] is not None else 1.0
    a = col["w_post"] * (1.0 if w["gate"] is None else torch.sigmoid(col["gate"]))
    rn = col["scale"] * r + a * (y * inv1)
    inv2 = torch.rsqrt(rn.pow(2).mean(-1, keepdim=True) + eps)
    dn = (col["w_pre"] * x["d_o"].double()).abs() if "d_o" in use and w["w_pre"] is not None else 0.0 * rn
    dR = (x["d_r"].double().abs() if "d_r" in use else 0.0) + inv2 * (dn + (rn * inv2).abs() * (dn * (rn * inv2).abs()).mean(-1, keepdim=True))
    size = lambda v: v.abs().amax(-1, keepdim=True)  # noqa: E731
    return size(col["scale"] * dR), size(inv1 * a * dR * (1 + (y * inv1) ** 2 if x["y"] is not None else 1.0))


def check(got, want, dtype, terms, amplitude=None, what=""):
    """|got - want| is at most the rounding of the result, plus fp32 arithmetic over `terms` summands: each
    fp32 operation is within 2^-24 of its operands' size, and sums that are formed along a fixed tree grow it by
    less than 4 sqrt(terms).  `amplitude`: size of the summands where they cancel."""
    if want is None:
        assert got is None
        return
    a = want.abs() if amplitude is None else torch.maximum(want.abs(), amplitude)
    bound = ROUND[dtype] * want.abs() * 1.001 + 2.0 ** -24 * (16 + 4 * math.sqrt(terms)) * a
    if dtype == "fp16":
        bound = bound + 2.0 ** -25            # results below the normal range
    bad = (got.double() - want).abs() > bound
    assert not bad.any(), (what, int(bad.sum()), float(((got.double() - want).abs() / bound).max()))


def run_and_check(x, w, dtype, eps=1e-6, use=("d_r", "d_o")):
    if w["w_pre"] is None:
        use = tuple(k for k in use if k != "d_o")
    r, o = B.residual_norm(x["y"], x["residual"], eps=eps, **w)
    want_r, want_o, g = exact(x, w, eps, use)
    n, d = want_r.shape[1:]
    size = want_r.pow(2).mean().sqrt()
    check(r, want_r, dtype, 1, size, "r'")
    check(o, want_o, dtype, d, None if want_o is None else want_o.pow(2).mean().sqrt(), "o")
    dy, dr, dw = B.residual_norm_backward(x["d_r"] if "d_r" in use else None, x["d_o"] if "d_o" in use else None,
                                          x["y"], x["residual"], eps=eps, **w)

    size_dr, size_dy = amplitudes(x, w, eps, use)
    check(dr, g["residual"], dtype, d, size_dr.expand_as(dr), "dr")
    if x["y"] is not None:
        check(dy, g["y"], dtype, d, size_dy.expand_as(dy), "dy")
    for name, t in zip(NAMES, dw):
        if w[name] is None:
            assert t is None
            continue
        want = g[name]
        if want is None:
            want = torch.zeros(t.shape, dtype=torch.float64, device="cuda")
        # the summands of a column: rows of size about that of the gradients times that of the values
        summand = 3.0 * math.sqrt(n) * 0.3
        check(t, want, dtype, d + n, torch.full_like(want, summand), name)
    assert B.operator_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("P,n,d", [(1, 1, 1), (2, 1, 8), (3, 5, 7), (1, 33, 64), (2, 17, 100), (5, 9, 129), (3, 64, 256), (1, 300, 264),
                                   (2, 41, 1000), (7, 3, 1001), (1, 5, 2048), (2, 9, 2056), (1, 11, 4095), (2, 6, 4096), (1, 4, 5001),
                                   (1, 3, 8192), (300, 2, 40)])
def test_forward_and_gradients(P, n, d, dtype):
    x, w = inputs(P, n, d, dtype)
    run_and_check(x, w, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d", [(3000, 96), (5000, 512), (1500, 1025)])
def test_many_rows(n, d, dtype):
    x, w = inputs(3, n, d, dtype, seed=1)
    run_and_check(x, w, dtype)


@pytest.mark.parametrize("given", [(), ("w_pre",), ("w_post",), ("gate",), ("scale",), ("w_post", "w_pre"), ("gate", "w_pre"),
                                   ("scale", "w_post", "gate")])
@pytest.mark.parametrize("d", [96, 333])
def test_what_is_not_given_drops_out(given, d):
    x, w = inputs(2, 19, d, "fp32", seed=2, given=given)
    run_and_check(x, w, "fp32")


def test_without_a_block_before_and_without_one_gradient():
    x, w = inputs(2, 19, 96, "fp32", seed=3, given=("scale", "w_pre"))
    x["y"] = None
    run_and_check(x, w, "fp32")
    run_and_check(x, w, "fp32", use=("d_o",))
    x, w = inputs(2, 19, 96, "bf16", seed=3)
    run_and_check(x, w, "bf16", use=("d_r",))
    run_and_check(x, w, "bf16", use=("d_o",))


@pytest.mark.parametrize("dtype,spread", [("bf16", 8), ("bf16", 3), ("fp32", 4), ("fp32", 1)])
def test_strides(dtype, spread):
    x, w = inputs(3, 23, 136, dtype, seed=4, spread=spread)
    run_and_check(x, w, dtype)


@pytest.mark.parametrize("shift", [1, 8])
def test_unaligned_views_of_a_buffer(shift):
    """Weights and gradients inside one [P, stride] buffer, activations that start off a 16-byte boundary."""
    P, n, d = 2, 9, 72
    x, w = inputs(P, n, d, "bf16", seed=5)
    for k, t in x.items():
        flat = torch.zeros(t.numel() + shift, dtype=t.dtype, device="cuda")
        x[k] = flat[shift:].view(P, n, d).copy_(t)
    grads = torch.full((P, 4 * d + 5), 3.0, dtype=torch.bfloat16, device="cuda")
    views = [grads[:, q * d + 1:(q + 1) * d + 1] for q in range(4)]
    run_and_check(x, w, "bf16")
    _, _, dw = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], d_weights=views, **w)
    _, _, plain = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    for a, b in zip(dw, plain):
        assert torch.equal(a, b)
    assert torch.all(grads[:, 0] == 3.0) and torch.all(grads[:, 4 * d + 1:] == 3.0)


def test_gradients_against_differences():
    P, n, d, eps = 1, 3, 24, 1e-5
    x, w = inputs(P, n, d, "fp32", seed=6)
    dy, dr, dw = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], eps=eps, **w)

    def loss(xx, ww):
        rms = lambda v: v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps)  # noqa: E731
        r = ww["scale"][:, None] * xx["residual"] + torch.sigmoid(ww["gate"])[:, None] * rms(xx["y"]) * ww["w_post"][:, None]
        return float((r * x["d_r"].double()).sum() + (rms(r) * ww["w_pre"][:, None] * x["d_o"].double()).sum())

    xd, wd = {k: v.double() for k, v in x.items()}, {k: v.double() for k, v in w.items()}
    h = 1e-5                                        # the difference's own error: h^2 times third derivatives
    for where, name, got in [(xd, "y", dy), (xd, "residual", dr)] + [(wd, k, g) for k, g in zip(NAMES, dw)]:
        for at in range(0, where[name].numel(), 5):
            flat = where[name].view(-1)
            keep = float(flat[at])
            flat[at] = keep + h
            up = loss(xd, wd)
            flat[at] = keep - h
            down = loss(xd, wd)
            flat[at] = keep
            assert abs((up - down) / (2 * h) - float(got.reshape(-1)[at])) < 2e-6, (name, at)


def test_rows_that_are_zero_infinite_or_not_numbers():
    """eps keeps a row of zeros finite; a bad row spoils its own results and its column sums only."""
    x, w = inputs(2, 6, 80, "fp32", seed=7)
    x["y"][0, 1] = 0
    x["residual"][0, 1] = 0
    run_and_check(x, w, "fp32")
    for value in (math.inf, math.nan):
        x["y"][1, 2, 5] = value
        r, o = B.residual_norm(x["y"], x["residual"], **w)
        dy, dr, dw = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
        ok = torch.ones((2, 6), dtype=torch.bool, device="cuda")
        ok[1, 2] = False
        for t in (r, o, dy, dr):
            assert torch.isfinite(t[ok]).all()
        assert not torch.isfinite(o[1, 2]).all()
        for t in dw[:2]:
            assert torch.isfinite(t[0]).all()


def test_in_place_streams_graph_and_repeatability():
    x, w = inputs(4, 50, 200, "bf16", seed=8)
    r, o = B.residual_norm(x["y"], x["residual"], **w)
    mine = x["residual"].clone()
    r2, o2 = B.residual_norm(x["y"], mine, residual_out=mine, **w)
    assert r2.data_ptr() == mine.data_ptr() and torch.equal(r2, r) and torch.equal(o2, o)
    first = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], stream=side, **w)
    side.synchronize()
    for a, b in zip((*first[:2], *first[2]), (*again[:2], *again[2])):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rg, og = B.residual_norm(x["y"], x["residual"], **w)
        back = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    x["y"].mul_(-1)
    graph.replay()
    torch.cuda.synchronize()
    want = B.residual_norm(x["y"], x["residual"], **w)
    assert torch.equal(rg, want[0]) and torch.equal(og, want[1])
    assert torch.equal(back[2][1], B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)[2][1])


def test_no_rows():
    x, w = inputs(2, 0, 64, "bf16")
    r, o = B.residual_norm(x["y"], x["residual"], **w)
    assert r.shape == o.shape == (2, 0, 64)
    dy, dr, dw = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    assert dy.shape == dr.shape == (2, 0, 64) and all(torch.all(t == 0) for t in dw)


def test_refusals():
    x, w = inputs(2, 4, 64, "fp32")
    bad = dict(w, w_post=w["w_post"][:, :-1])
    for call in (lambda: B.residual_norm(x["y"], x["residual"], **bad),
                 lambda: B.residual_norm(x["y"][:1], x["residual"], **w),
                 lambda: B.residual_norm(x["y"].bfloat16(), x["residual"], **w),
                 lambda: B.residual_norm(x["y"].cpu(), x["residual"], **w),
                 lambda: B.residual_norm(x["y"], x["residual"][0], **w),
                 lambda: B.residual_norm(x["y"], x["residual"].double(), **w),
                 lambda: B.residual_norm(x["y"].transpose(1, 2).contiguous().transpose(1, 2), x["residual"], **w),
                 lambda: B.residual_norm(None, x["residual"], **w),                       # a gate without a block
                 lambda: B.residual_norm(x["y"], x["residual"], eps=-1.0, **w),
                 lambda: B.residual_norm(x["y"], x["residual"], eps=math.nan, **w),
                 lambda: B.residual_norm(x["y"], x["residual"], residual_out=x["residual"][:, :1].expand(2, 4, 64), **w),
                 lambda: B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], w_post=w["w_post"]),   # d_out without w_pre
                 lambda: B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], d_weights=(None,), **w),
                 lambda: B.residual_norm(torch.zeros(1, 1, 8193, device="cuda"), torch.zeros(1, 1, 8193, device="cuda")),
                 lambda: B.residual_norm(x["y"].cpu(), x["residual"].cpu())):
        with pytest.raises(B.EventGradError):
            call()
    lib = B.load_library()
    assert lib.eg_residual_norm(None, None) == 1 and lib.eg_residual_norm_backward(None, None) == 1
    assert lib.eg_residual_norm_workspace(0, 64) == 0 and lib.eg_residual_norm_workspace(2, 8193) == 0
