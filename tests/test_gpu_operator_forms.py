"""Forms of the operators that leave something out, and values at the ends of their ranges, at the sizes where each kernel
takes them, against the formulas in 64 bits."""
import pytest
import torch

import test_gpu_feed_forward as F
import test_gpu_residual_norm as N
from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu


def forward_again_and_again(x, w, dtype, turns=8):
    """The forward call against the formula, and the same bits every time."""
    want_r, want_o, _ = N.exact(x, w, 1e-6, use=("d_r",))
    d = want_r.shape[2]
    first = B.residual_norm(x["y"], x["residual"], **w)
    N.check(first[0], want_r, dtype, 1, want_r.pow(2).mean().sqrt(), "r'")
    N.check(first[1], want_o, dtype, d, None if want_o is None else want_o.pow(2).mean().sqrt(), "o")
    for _ in range(turns):
        for a, b in zip(B.residual_norm(x["y"], x["residual"], **w), first):
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(2, 1024, 1024), (4, 1100, 512), (1, 1100, 4096), (2, 700, 2048), (3, 500, 1001)])
@pytest.mark.parametrize("given", [("w_post",), ("w_pre",), ("gate", "scale", "w_pre"), ("w_post", "gate", "scale")])
def test_norm_of_some_thousand_rows_with_one_of_the_two_norms(given, P, n, d, dtype):
    """Several rows a group of warps, one sum a row: the buffer of a row's sums is not the one before's."""
    x, w = N.inputs(P, n, d, dtype, seed=21, given=given)
    forward_again_and_again(x, w, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(2, 1024, 1024), (1, 1100, 4096), (3, 500, 1001)])
def test_norm_of_some_thousand_rows_without_a_block_before(P, n, d, dtype):
    x, w = N.inputs(P, n, d, dtype, seed=22, given=("scale", "w_pre"))
    x["y"] = None
    forward_again_and_again(x, w, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(1, 900, 1001), (3, 220, 333), (1, 1184, 4095), (2, 500, 777)])
@pytest.mark.parametrize("given", [("w_post",), ("w_pre",), ("gate", "scale", "w_pre"), ("w_post", "gate", "scale")])
def test_norm_of_unaligned_rows_two_a_block_with_one_of_the_two_norms(given, P, n, d, dtype):
    x, w = N.inputs(P, n, d, dtype, seed=23, given=given)
    forward_again_and_again(x, w, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(1, 200, 1024), (2, 140, 4096), (1, 290, 1001), (5, 50, 640)])
@pytest.mark.parametrize("given", [(), ("w_pre",), ("scale", "w_pre"), ("gate", "scale", "w_pre")])
def test_norm_gradients_of_two_rows_a_block_without_the_first_norm(given, P, n, d, dtype):
    x, w = N.inputs(P, n, d, dtype, seed=24, given=given)
    N.run_and_check(x, w, dtype)
    call = lambda: B.residual_norm_backward(x["d_r"], x["d_o"] if "w_pre" in given else None, x["y"], x["residual"], **w)  # noqa: E731
    first = call()
    for _ in range(8):
        again = call()
        for a, b in zip((*first[:2], *first[2]), (*again[:2], *again[2])):
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(2, 701, 96), (2, 701, 1024), (1, 1101, 4096), (3, 333, 513), (1, 301, 5000), (2, 60, 96)])
@pytest.mark.parametrize("given", [N.NAMES, ("w_pre",), ("w_post", "gate")])
def test_norm_without_an_epsilon(given, P, n, d, dtype):
    """eps = 0 is defined for rows that are not zero, however many rows the last step of a run holds."""
    x, w = N.inputs(P, n, d, dtype, seed=25, given=given)
    N.run_and_check(x, w, dtype, eps=0.0)


@pytest.mark.parametrize("given", [N.NAMES, ("w_pre",), ("w_post",)])
def test_norm_without_an_epsilon_keeps_zero_rows_to_themselves(given):
    """0 / 0 in its own row and replica, nowhere else."""
    x, w = N.inputs(3, 333, 96, "fp32", seed=26, given=given)
    args = lambda: (x["d_r"], x["d_o"] if "w_pre" in given else None, x["y"], x["residual"])  # noqa: E731
    clean = B.residual_norm_backward(*args(), eps=0.0, **w)
    x["y"][1, 7] = 0
    x["residual"][1, 7] = 0
    got = B.residual_norm_backward(*args(), eps=0.0, **w)
    rows = torch.ones(3, 333, dtype=torch.bool, device="cuda")
    rows[1, 7] = False
    for a, b in zip(got[:2], clean[:2]):
        assert torch.equal(a[rows], b[rows])
    for a, b in zip(got[2], clean[2]):
        assert a is None or torch.equal(a[[0, 2]], b[[0, 2]])


SUMS_BEYOND = [(2, 33, 1024), (2, 200, 1024), (2, 3000, 1024), (1, 2500, 96), (1, 1200, 4104), (2, 700, 1001)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", SUMS_BEYOND)
def test_norm_where_the_squares_of_a_block_pass_32_bits(P, n, d, dtype):
    """A sum of squares that is infinite in 32 bits makes rms(y) zero, in every kernel: r' = scale * r and what follows from it."""
    x, w = N.inputs(P, n, d, dtype, seed=27)
    none = dict(x, y=torch.zeros_like(x["y"]))
    want_r, want_o, g = N.exact(none, w, 1e-6)
    x["y"] = torch.where(x["y"] > 0, 5e18, -5e18).to(N.TYPES[dtype])       # 96 squares of them: 2.4e39
    r, o = B.residual_norm(x["y"], x["residual"], **w)
    N.check(r, want_r, dtype, 1, want_r.pow(2).mean().sqrt(), "r'")
    N.check(o, want_o, dtype, d, want_o.pow(2).mean().sqrt(), "o")
    dy, dr, dw = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    N.check(dr, g["residual"], dtype, d, N.amplitudes(none, w, 1e-6, ("d_r", "d_o"))[0].expand_as(dr), "dr")
    assert torch.all(dy == 0) and torch.all(dw[0] == 0) and torch.all(dw[1] == 0)
    for name, t in list(zip(N.NAMES, dw))[2:]:
        N.check(t, g[name], dtype, d + n, torch.full_like(g[name], 0.9 * n ** 0.5), name)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", SUMS_BEYOND)
def test_norm_where_only_the_weighted_squares_pass_32_bits(P, n, d, dtype):
    """(a y)^2 passes the range of 32 bits, y^2 and r'^2 do not."""
    x, w = N.inputs(P, n, d, dtype, seed=28, given=("w_post", "scale", "w_pre"))
    x["y"] = (x["y"].float() * 3e16).to(N.TYPES[dtype])
    w["w_post"] = (w["w_post"].float() * 256).to(N.TYPES[dtype])
    N.run_and_check(x, w, dtype)


def products_alone(x, w):
    """x w^T of the tiles' kernel by itself: with relu, U = 1 and a projection that is a piece of the unit matrix, y = G."""
    P, n, d = x.shape
    f = w.shape[1]
    x[..., 0] = 1.0
    w_up = torch.zeros(P, f, d, device="cuda")
    w_up[..., 0] = 1.0
    w_down = torch.eye(d, f, device="cuda").expand(P, d, f).contiguous()
    k = min(d, f)
    y, _ = B.feed_forward(x, w, w_up, w_down, activation="relu", save=True)
    return y[..., :k], (x.double() @ w.double().transpose(1, 2))[..., :k]


@pytest.mark.parametrize("kind", ["worst", "random"])
@pytest.mark.parametrize("d", [16, 64, 256, 1024])
def test_products_of_fp32_parts(kind, d):
    """Positive values, so that errors of one sign show.  In units u = 2^-23 of the sum: parts left out 1/2; an addition into the
    accumulator of the first parts truncates by one of what it holds so far (d / 16 of them grow to the sum, at most 16
    at a time); their sums are added in 32 bits, 1/2 each of what there is; the accumulator of the smaller parts holds 2^-7 and meets
    5 d / 16 additions; the last addition 1/2."""
    worst = torch.tensor([0x3f80ffff], dtype=torch.int32).view(torch.float32).item()     # parts by truncation: 2^-7 and 2^-15 left
    gen = torch.Generator(device="cuda").manual_seed(29)
    make = lambda *s: torch.full(s, worst, device="cuda") if kind == "worst" else 1 + torch.rand(s, generator=gen, device="cuda")  # noqa: E731
    y, want = products_alone(make(1, 300, d), make(1, 128, d))
    adds = max(1, d // 16)
    chunks = -(-adds // 16)
    units = 0.5 + (min(adds, 16) + 1) / 2 + (chunks + 1) / 4 * (chunks > 1) + 5 * adds / 2 * 2 ** -7 + 0.5
    assert float(((y.double() - want) / want).abs().max()) <= units * 2.0 ** -23


def test_products_of_fp32_values_near_the_ends_of_their_range():
    """The largest finite values keep their parts (rounded to bf16 they would be infinite); the smallest ones lose at most what
    bf16 cannot hold."""
    top = torch.finfo(torch.float32).max
    x = torch.zeros(1, 70, 16, device="cuda")
    w = torch.zeros(1, 16, 16, device="cuda")
    w[0, :, 1] = 0.5
    values = [top, top * (1 - 2.0 ** -9), 3.39e38, 3.4e38, 1e38, 2.0 ** -100, 1.7e-33, 2.0 ** -126]
    for i, v in enumerate(values):
        x[0, i, 1] = v
    y, want = products_alone(x, w)
    assert torch.all((y.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -133)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 8, 40, 300])
def test_an_infinite_operand_has_one_result_in_every_kernel(n, dtype):
    """Positive operands: infinity times any of them is infinity, whatever kernel the number of tokens goes to and whether or not
    the other has smaller parts."""
    d, f, dt = 64, 96, N.TYPES[dtype]
    full = lambda rows, cols, v: torch.full((1, rows, cols), v, device="cuda").to(dt)  # noqa: E731
    for value in (0.5, 0.3):                          # one part, three parts
        w = (full(f, d, value), full(f, d, value), full(d, f, value))
        x = full(n, d, 1.0)
        x[0, 0, 3] = float("inf")
        alone = B.feed_forward(x, *w)
        y, saved = B.feed_forward(x, *w, save=True)
        for got in (alone, y):
            assert torch.all(torch.isposinf(got[0, 0])) and torch.isfinite(got[0, 1:]).all()
        x[0, 0, 3] = 1.0
        dy = full(n, d, 0.25)
        dy[0, 0, 5] = float("inf")
        _, saved = B.feed_forward(x, *w, save=True)
        dx, (d_gate, d_up, d_down) = B.feed_forward_backward(dy, x, *w, saved)
        assert torch.all(torch.isposinf(dx[0, 0])) and torch.isfinite(dx[0, 1:]).all()
        assert torch.all(torch.isposinf(d_gate)) and torch.all(torch.isposinf(d_up)) and torch.all(torch.isposinf(d_down[0, 5]))
        assert torch.isfinite(d_down[0, 6:]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("P,n,d,f", [(3, 1, 64, 96), (2, 9, 64, 96), (3, 45, 64, 104), (2, 300, 264, 136), (3, 5, 33, 51), (2, 70, 41, 66)])
@pytest.mark.parametrize("room", [0, 8])
def test_feed_forward_of_replicas_that_take_turns_row_by_row(P, n, d, f, room, dtype):
    """[rows][P][columns]: the same bits as one replica after the other, and nothing between the rows is written."""
    t = F.inputs(P, n, d, f, dtype, seed=30)
    names = ("x", "w_gate", "w_up", "w_down", "dy")

    def in_turn(m, fill):
        to = torch.full((m.shape[1], P, m.shape[2] + room), fill, dtype=m.dtype, device="cuda")
        to[..., :m.shape[2]] = m.transpose(0, 1)
        return to

    x, wg, wu, wd, dy = (in_turn(t[k], 7.0)[..., :t[k].shape[2]].transpose(0, 1) for k in names)
    buffers = [in_turn(torch.full_like(t[k], 3.0), 3.0) for k in ("x", "w_gate", "w_up", "w_down")]
    out, *grads = (b[..., :t[k].shape[2]].transpose(0, 1) for b, k in zip(buffers, names))
    want = F.run(t, "silu")
    assert torch.equal(B.feed_forward(x, wg, wu, wd), want["alone"])
    y, saved = B.feed_forward(x, wg, wu, wd, save=True, out=out)
    dx, _ = B.feed_forward_backward(dy, x, wg, wu, wd, saved, d_weights=grads)
    for name, got in zip(F.NAMES, (y, dx, *grads)):
        assert torch.equal(got, want[name]), name
    for b, k in zip(buffers, names):
        assert torch.all(b[..., t[k].shape[2]:] == 3.0)
    assert B.operator_status() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(3, 5, 64), (2, 700, 96), (2, 9, 33), (4, 2, 8)])
@pytest.mark.parametrize("room", [0, 8])
def test_norm_of_replicas_that_take_turns_row_by_row(P, n, d, room, dtype):
    x, w = N.inputs(P, n, d, dtype, seed=31)
    want = B.residual_norm(x["y"], x["residual"], **w)
    back = B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)
    buffers = [torch.full((n, P, d + room), 3.0, dtype=N.TYPES[dtype], device="cuda") for _ in range(6)]
    views = [b[..., :d].transpose(0, 1) for b in buffers]
    for v, k in zip(views, ("y", "residual", "d_r", "d_o")):
        v.copy_(x[k])
    y, r, d_r, d_o, r_out, out = views
    got = B.residual_norm(y, r, residual_out=r_out, out=out, **w)
    assert got[0].data_ptr() == r_out.data_ptr()
    size = {"fp32": 2.0 ** -20, "bf16": 2.0 ** -6}[dtype]             # another kernel may take other strides: other sums, one unit
    for a, b in zip((*got, *B.residual_norm_backward(d_r, d_o, y, r, **w)[:2]), (*want, *back[:2])):
        assert torch.all((a.double() - b.double()).abs() <= size * b.double().abs().amax(-1, keepdim=True))
    for b in buffers:
        assert torch.all(b[..., d:] == 3.0)


def test_a_wait_that_runs_out_is_reported_once_and_leaves_the_device_usable():
    assert B.operator_status() == 0
    x, w = N.inputs(2, 400, 512, "bf16", seed=32)
    want = B.residual_norm(x["y"], x["residual"], **w)
    for which in (0, 1, 2):
        B.selftest_operator_wait(which)
        assert B.operator_status() == 5               # EG_ERR_TIMEOUT
        assert B.operator_status() == 0
        for a, b in zip(B.residual_norm(x["y"], x["residual"], **w), want):
            assert torch.equal(a, b)
    t = F.inputs(2, 40, 64, 96, "bf16", seed=32)
    F.run_and_check(t, "bf16")
    for which in (-1, 3):
        with pytest.raises(B.EventGradError):
            B.selftest_operator_wait(which)


def test_tensors_that_require_gradients_are_refused():
    """The operators take no part in autograd: no result without a graph where one is expected."""
    x, w = N.inputs(2, 5, 64, "fp32", seed=33)
    t = F.inputs(2, 5, 64, 96, "fp32", seed=33)
    weights = (t["w_gate"], t["w_up"], t["w_down"])
    y, saved = B.feed_forward(t["x"], *weights, save=True)
    eg = B.EventGrad(2, [40])
    g = torch.ones(2, eg.replica_stride, device="cuda")

    def calls(leaf):
        swap = lambda m: m.requires_grad_() if m is leaf else m  # noqa: E731
        norm = {k: swap(v) for k, v in w.items()}
        ffn = [swap(m) for m in weights]
        yield (x["y"], x["residual"], *w.values()), lambda: B.residual_norm(swap(x["y"]), swap(x["residual"]), **norm)[1]
        yield (x["d_r"], x["d_o"], x["y"], x["residual"], *w.values()), lambda: B.residual_norm_backward(
            swap(x["d_r"]), swap(x["d_o"]), swap(x["y"]), swap(x["residual"]), **norm)[0]
        yield (t["x"], *weights), lambda: B.feed_forward(swap(t["x"]), *ffn)
        yield (t["dy"], t["x"], *weights), lambda: B.feed_forward_backward(swap(t["dy"]), swap(t["x"]), *ffn, saved)[0]
        yield (g,), lambda: eg.clip_gradients(swap(g), 1e9)

    for number in range(5):
        tensors, call = list(calls(None))[number]
        want = call()
        for leaf in tensors:
            _, call = list(calls(leaf))[number]
            with pytest.raises(B.EventGradError, match="autograd"):
                call()
            with torch.no_grad():
                assert torch.equal(call(), want)
            leaf.requires_grad_(False)


@pytest.mark.parametrize("n", [1, 5, 40, 300])
def test_values_between_the_products_have_the_range_of_the_type(n):
    """H passes 65504 in fp16, y would not: infinite in every kernel, and never another number; bf16 has the range."""
    d, f = 64, 96
    for dtype, infinite in (("fp16", True), ("bf16", False), ("fp32", False)):
        full = lambda rows, cols, v: torch.full((1, rows, cols), v, device="cuda").to(N.TYPES[dtype])  # noqa: E731
        w = (full(f, d, 2.0), full(f, d, 2.0), full(d, f, 2.0 ** -12))
        x = full(n, d, 4.0)                                  # G = U = 512, H = 2^18, y = 6144
        y, saved = B.feed_forward(x, *w, save=True)
        for got in (y, B.feed_forward(x, *w)):
            assert torch.all(torch.isposinf(got) if infinite else got == 6144.0)
