"""The gated feed-forward block of every replica and its gradients against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
#: Half a unit in the last place, relative: 8 and 11 significant bits; fp32 intermediates are not rounded further.
ROUND = {"fp32": 0.0, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
NAMES = ("y", "dx", "d_gate", "d_up", "d_down")


def inputs(P, n, d, f, dtype, seed=0, spread=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]

    def make(rows, cols, scale):
        t = torch.randn((P, rows, cols + spread), generator=gen, device="cuda") * scale
        return t.to(dt)[:, :, :cols]

    return dict(x=make(n, d, 1.0), w_gate=make(f, d, d ** -0.5), w_up=make(f, d, d ** -0.5), w_down=make(d, f, f ** -0.5),
                dy=make(n, d, 0.2))


def act_of(name, g):
    """act, act' and a bound of |act''|"""
    if name == "relu":
        return torch.relu(g), (g > 0).double(), 0.0
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), 0.5
    cdf = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 0.8


def exact(t, act):
    """The results in 64 bits, and how far a computation may be from each element: every product of two
    matrices is off by at most e times the product of their absolute values (tensor-core sums truncate: one unit of
    2^-23 per instruction of 16 elements, over a run of at most 16 instructions in fp32 and over the whole of K
    else), every value that is rounded to 16 bits by u of itself; the rest follows to first order, and
    5 % are added for the higher orders."""
    x, wg, wu, wd, dy = (t[k].double() for k in ("x", "w_gate", "w_up", "w_down", "dy"))
    dtype = {v: k for k, v in TYPES.items()}[t["x"].dtype]
    u = ROUND[dtype]
    T = lambda m: m.transpose(1, 2)  # noqa: E731

    def prod(a, b, ea, eb):
        """(a b, its error) from matrices that are off by ea, eb"""
        k = a.shape[2]
        e = 2.0 ** -19 if dtype == "fp32" else (k / 16 + 1) * 2.0 ** -23
        err = e * (a.abs() @ b.abs())
        if ea is not None:
            err = err + ea @ b.abs()
        if eb is not None:
            err = err + a.abs() @ eb
        return a @ b, err

    g, eg = prod(x, T(wg), None, None)
    up, eu = prod(x, T(wu), None, None)
    a, da, dda = act_of(act, g)
    h = a * up
    f32 = 2.0 ** -22                                     # the activation's own fp32 arithmetic
    eh = (da * up).abs() * eg + a.abs() * eu + (u + f32) * (h.abs() + g.abs() * up.abs())
    y, ey = prod(h, T(wd), eh, None)
    dh, edh = prod(dy, wd, None, None)
    eg, eu = eg + u * g.abs(), eu + u * up.abs()          # as the backward pass reads them
    du, dg = dh * a, dh * up * da
    edu = edh * a.abs() + dh.abs() * (da.abs() * eg) + (u + f32) * (du.abs() + (dh * g).abs())
    edg = edh * (up * da).abs() + dh.abs() * (da.abs() * eu + up.abs() * dda * eg) + (u + f32) * (dg.abs() + (dh * up).abs())
    dx1, e1 = prod(dg, wg, edg, None)
    dx2, e2 = prod(du, wu, edu, None)
    dwg, ewg = prod(T(dg), x, T(edg), None)
    dwu, ewu = prod(T(du), x, T(edu), None)
    dwd, ewd = prod(T(dy), h, None, eh)
    out = {"y": (y, ey), "dx": (dx1 + dx2, e1 + e2), "d_gate": (dwg, ewg), "d_up": (dwu, ewu), "d_down": (dwd, ewd)}
    last = max(u, 2.0 ** -24)
    return {k: (v, 1.05 * (e + last * v.abs()) + (2.0 ** -25 if dtype == "fp16" else 1e-30)) for k, (v, e) in out.items()}


def check(got, want, dtype, names=NAMES):
    u = ROUND[dtype]
    for k in names:
        v, bound = want[k]
        far = (got[k].double() - v).abs()
        assert torch.all(far <= bound), (k, float((far / bound).max()))
        # over all elements: roundings are independent, each of at most u / sqrt(3) in the mean; y and d_down meet two of
        # them, the others up to four, one of them with a factor of 1.5; fp32: three products in a row
        most = {"fp32": 3.5e-6}.get(dtype, u * (1.0 if k in ("y", "d_down") else 1.5))
        if v.numel() > 64:
            assert float(far.norm()) <= most * float(v.norm()), (k, float(far.norm() / v.norm()))


def run(t, act, **kw):
    w = (t["w_gate"], t["w_up"], t["w_down"])
    y, saved = B.feed_forward(t["x"], *w, activation=act, save=True)
    dx, dw = B.feed_forward_backward(t["dy"], t["x"], *w, saved, activation=act, **kw)
    alone = B.feed_forward(t["x"], *w, activation=act)
    assert B.operator_status() == 0
    return dict(zip(NAMES, (y, dx, *dw)), alone=alone)


def run_and_check(t, dtype, act="silu"):
    got, want = run(t, act), exact(t, act)
    check(got, want, dtype)
    check(dict(y=got["alone"]), want, dtype, ("y",))


SIZES = [(1, 1, 1, 1), (1, 1, 8, 8), (2, 3, 5, 7), (1, 128, 64, 64), (3, 1, 72, 200), (2, 17, 40, 24), (1, 33, 257, 130), (2, 130, 64, 300),
         (1, 255, 96, 256), (1, 257, 520, 136), (5, 64, 33, 129), (1, 600, 128, 384), (2, 31, 1000, 72), (40, 3, 16, 24)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("P,n,d,f", SIZES)
def test_block_and_gradients(P, n, d, f, dtype):
    run_and_check(inputs(P, n, d, f, dtype), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "relu"])
@pytest.mark.parametrize("P,n,d,f", [(2, 37, 64, 96), (1, 5, 19, 33)])
def test_activations(P, n, d, f, dtype, act):
    run_and_check(inputs(P, n, d, f, dtype, seed=1), dtype, act)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 16, 17, 40])
def test_few_tokens(n, dtype):
    """Answering: one token or a few."""
    for d, f in ((256, 1024), (136, 330), (101, 77)):
        t = inputs(2, n, d, f, dtype, seed=n)
        y = B.feed_forward(t["x"], t["w_gate"], t["w_up"], t["w_down"])
        check(dict(y=y), exact(t, "silu"), dtype, ("y",))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_more_tiles_than_multiprocessors(dtype):
    run_and_check(inputs(3, 700, 320, 1100, dtype, seed=2), dtype)


@pytest.mark.parametrize("dtype,spread", [("bf16", 8), ("bf16", 1), ("fp16", 24), ("fp32", 4), ("fp32", 3)])
def test_strides(dtype, spread):
    run_and_check(inputs(2, 45, 64, 104, dtype, seed=3, spread=spread), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,f", [(64, 96), (37, 51)])
def test_weights_and_gradients_in_the_layout_of_the_step(dtype, d, f):
    P, n, dt = 3, 20, TYPES[dtype]
    eg = B.EventGrad(P, [d, f * d, 5, f * d, d * f])
    params = torch.zeros((P, eg.replica_stride), dtype=dt, device="cuda")
    grads = torch.full_like(params, 3.0)
    t = inputs(P, n, d, f, dtype, seed=4)
    shapes = {1: (f, d), 3: (f, d), 4: (d, f)}
    for q, k in ((1, "w_gate"), (3, "w_up"), (4, "w_down")):
        v = eg.view(params, q, shapes[q])
        v.copy_(t[k])
        t[k] = v
    got = run(t, "silu", d_weights=[eg.view(grads, q, shapes[q]) for q in (1, 3, 4)])
    check(got, exact(t, "silu"), dtype)
    for q in (0, 2):
        assert torch.all(grads[:, eg.tensor_offset[q]:eg.tensor_offset[q] + eg.numel[q]] == 3.0)
    covered = torch.zeros_like(grads, dtype=torch.bool)
    for o, m in zip(eg.tensor_offset, eg.numel):
        covered[:, o:o + m] = True
    assert torch.all(grads[~covered] == 3.0), "padding was written"


def test_some_gradients_only():
    t = inputs(2, 30, 64, 128, "bf16", seed=5)
    w = (t["w_gate"], t["w_up"], t["w_down"])
    _, saved = B.feed_forward(t["x"], *w, save=True)
    full = B.feed_forward_backward(t["dy"], t["x"], *w, saved)
    down = torch.empty_like(t["w_down"])
    dx, dw = B.feed_forward_backward(t["dy"], t["x"], *w, saved, d_weights=(None, None, down))
    assert torch.equal(dx, full[0]) and dw[0] is None and torch.equal(down, full[1][2])


def test_gradients_against_differences():
    t = inputs(1, 4, 12, 20, "fp32", seed=6)
    got = run(t, "gelu")
    td = {k: v.double().clone() for k, v in t.items()}

    def loss():
        a = act_of("gelu", td["x"] @ td["w_gate"].transpose(1, 2))[0]
        return float((((a * (td["x"] @ td["w_up"].transpose(1, 2))) @ td["w_down"].transpose(1, 2)) * td["dy"]).sum())

    h = 1e-5                                      # the difference's own error is of order h^2
    for name, grad in (("x", "dx"), ("w_gate", "d_gate"), ("w_up", "d_up"), ("w_down", "d_down")):
        flat = td[name].view(-1)
        for at in range(0, flat.numel(), 7):
            keep = float(flat[at])
            flat[at] = keep + h
            up = loss()
            flat[at] = keep - h
            down = loss()
            flat[at] = keep
            assert abs((up - down) / (2 * h) - float(got[grad].reshape(-1)[at])) < 2e-6, (name, at)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinities_and_nan_stay_in_their_rows(dtype):
    t = inputs(2, 40, 64, 96, dtype, seed=7)
    clean = run(t, "silu")
    for value in (math.inf, math.nan):
        t["x"][1, 7, 3] = value
        got = run(t, "silu")
        rows = torch.ones((2, 40), dtype=torch.bool, device="cuda")
        rows[1, 7] = False
        assert torch.equal(got["y"][rows], clean["y"][rows]) and torch.equal(got["dx"][rows], clean["dx"][rows])
        assert not torch.isfinite(got["y"][1, 7]).any()
        assert torch.equal(got["d_gate"][0], clean["d_gate"][0])


def test_same_bits_on_another_stream_and_in_a_graph():
    t = inputs(2, 300, 128, 256, "bf16", seed=8)
    w = (t["w_gate"], t["w_up"], t["w_down"])
    first = run(t, "silu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, saved = B.feed_forward(t["x"], *w, save=True, stream=side)
    dx, dw = B.feed_forward_backward(t["dy"], t["x"], *w, saved, stream=side)
    side.synchronize()
    for k, v in zip(NAMES, (y, dx, *dw)):
        assert torch.equal(first[k], v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, saved = B.feed_forward(t["x"], *w, save=True)
        dx, dw = B.feed_forward_backward(t["dy"], t["x"], *w, saved)
    t["x"].mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    again = run(t, "silu")
    for k, v in zip(NAMES, (y, dx, *dw)):
        assert torch.equal(again[k], v)


def test_no_rows():
    t = inputs(2, 0, 64, 33, "bf16")
    got = run(t, "silu")
    assert got["y"].shape == got["dx"].shape == (2, 0, 64)
    assert all(torch.all(got[k] == 0) for k in NAMES[2:])


def test_refusals():
    t = inputs(2, 4, 16, 24, "bf16")
    x, w = t["x"], (t["w_gate"], t["w_up"], t["w_down"])
    _, saved = B.feed_forward(x, *w, save=True)
    for call in (lambda: B.feed_forward(x, w[0], w[1], w[0]),
                 lambda: B.feed_forward(x[:1], *w),
                 lambda: B.feed_forward(x, w[0].float(), *w[1:]),
                 lambda: B.feed_forward(x.double(), *(m.double() for m in w)),
                 lambda: B.feed_forward(x[0], *w),
                 lambda: B.feed_forward(x, *w, activation="tanh"),
                 lambda: B.feed_forward(x, w[0].transpose(1, 2).contiguous().transpose(1, 2), *w[1:]),
                 lambda: B.feed_forward(x, *w, out=torch.empty(2, 4, 17, dtype=x.dtype, device="cuda")),
                 lambda: B.feed_forward(x[:1].expand(2, 4, 16), *w),                    # replicas on one another
                 lambda: B.feed_forward(x.cpu(), *(m.cpu() for m in w)),
                 lambda: B.feed_forward_backward(t["dy"], x, *w, saved[:100]),
                 lambda: B.feed_forward_backward(t["dy"], x, *w, saved.float()),
                 lambda: B.feed_forward_backward(t["dy"][:, :2], x, *w, saved),
                 lambda: B.feed_forward_backward(t["dy"], x, *w, saved, d_weights=(None,))):
        with pytest.raises(B.EventGradError):
            call()
    lib = B.load_library()
    assert lib.eg_feed_forward(None, None, 0, None) == 1 and lib.eg_feed_forward_backward(None, None, 0, None) == 1
    assert lib.eg_feed_forward_workspace(None, 0) == 0 and lib.eg_feed_forward_saved_bytes(None) == 0
