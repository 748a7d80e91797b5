"""The embedding of tokens and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
#: Half a unit in the last place of a result, relative (24, 8 and 11 significant bits), and half a step below fp16's normal range.
ROUND = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 0.0, "bf16": 0.0, "fp16": 2.0 ** -25}


def inputs(P, n, V, d, dtype, seed=0, outside=0.2, bits=64):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand((P, n), generator=gen, device="cuda", dtype=torch.float64)
    tokens = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp_(0, V - 1)
    odd = torch.rand((P, n), generator=gen, device="cuda") < outside
    far = torch.tensor([-1, V, -V, 2 ** 31 - 1, -2 ** 31] + ([2 ** 40, -2 ** 62] if bits == 64 else []), device="cuda")
    tokens = torch.where(odd, far[torch.randint(0, len(far), (P, n), generator=gen, device="cuda")], tokens)
    w = torch.randn((P, V, d), generator=gen, device="cuda").to(TYPES[dtype])
    dy = torch.randn((P, n, d), generator=gen, device="cuda").to(TYPES[dtype])
    return (tokens.int() if bits == 32 else tokens), w, dy


def check_forward(y, tokens, w, scale, dtype):
    P, n = tokens.shape
    V = w.shape[1]
    inside = (tokens >= 0) & (tokens < V)
    rows = w[torch.arange(P, device="cuda")[:, None], tokens.long().clamp(0, V - 1)].double() * scale
    want = torch.where(inside[:, :, None], rows, torch.zeros_like(rows))
    # scale and product round in 32 bits
    assert ((y.double() - want).abs() <= (ROUND[dtype] * 1.001 + 2.0 ** -23) * want.abs() + TINY[dtype]).all()
    assert (y[~inside] == 0).all()


def gradient(tokens, dy, V, scale):
    """(gradient, sum of the summands' sizes, number of summands) in 64 bits."""
    P, n, d = dy.shape
    want, size, count = (torch.zeros((P, V, k), dtype=torch.float64, device="cuda") for k in (d, d, 1))
    for i in range(P):
        at = torch.nonzero((tokens[i] >= 0) & (tokens[i] < V))[:, 0]
        t, g = tokens[i, at].long(), dy[i, at].double()
        want[i].index_add_(0, t, g * scale)
        size[i].index_add_(0, t, (g * scale).abs())
        count[i].index_add_(0, t, torch.ones_like(g[:, :1]))
    return want, size, count


def check_gradient(got, tokens, dy, scale, dtype, before=None):
    want, size, count = gradient(tokens, dy, got.shape[1], scale)
    # each of the sums, the scale, its product (and the sum with what was there) rounds in 32 bits
    steps = count + 3
    if before is not None:
        want, size = want + before.double(), size + before.double().abs()
    bound = ROUND[dtype] * 1.001 * want.abs() + 2.0 ** -24 * steps * size + TINY[dtype]
    bad = (got.double() - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), float((got.double() - want).abs().max()))
    none = (count == 0)[:, :, 0]
    assert (got[none] == (0 if before is None else before[none])).all()


SIZES = [(1, 1, 1, 1), (4, 1, 1000, 64), (2, 31, 7, 33), (1, 32, 40, 8), (3, 777, 1009, 509), (2, 5000, 300, 96), (1, 40000, 50, 24),
         (2, 2048, 70000, 8), (5, 333, 513, 1032), (1, 65, 64, 4104)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("P,n,V,d", SIZES)
def test_sizes(P, n, V, d, dtype):
    tokens, w, dy = inputs(P, n, V, d, dtype, bits=32 if n % 2 else 64)
    y = B.embedding(tokens, w, scale=1.7)
    check_forward(y, tokens, w, 1.7, dtype)
    got = B.embedding_backward(dy, tokens, vocabulary=V, scale=1.7)
    check_gradient(got, tokens, dy, 1.7, dtype)
    assert torch.equal(got, B.embedding_backward(dy, tokens, vocabulary=V, scale=1.7))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [40, 41])
@pytest.mark.parametrize("kind", ["one", "last", "none", "sorted", "back", "two", "ends"])
def test_ways_the_tokens_come(kind, d, dtype):
    """One token in every place (its run crosses every chunk), none of the table's, sorted, two that alternate, only the table's
    first and last row."""
    P, n, V = 2, 2500, 600
    tokens, _, dy = inputs(P, n, V, d, dtype, outside=0.0)
    at = torch.arange(n, device="cuda").expand(P, n)
    tokens = {"one": torch.full_like(tokens, 37), "last": torch.where(at < n - 1, -1, 599), "none": torch.full_like(tokens, -1),
              "sorted": tokens.sort(1)[0], "back": tokens.sort(1, descending=True)[0], "two": at % 2 * 599, "ends": at // 1250 * 599}[kind]
    got = B.embedding_backward(dy, tokens, vocabulary=V)
    check_gradient(got, tokens, dy, 1.0, dtype)


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 1023, 1024, 1025])
def test_runs_that_end_where_chunks_do(n):
    tokens, _, dy = inputs(1, n, 4, 16, "fp32", outside=0.0)
    for run in (1, 31, 32, 33, 64, 96):
        t = (torch.arange(n, device="cuda") // run % 4)[None]
        check_gradient(B.embedding_backward(dy, t, vocabulary=4), t, dy, 1.0, "fp32")


@pytest.mark.parametrize("dtype", list(TYPES))
def test_adds_to_what_is_there(dtype):
    tokens, w, dy = inputs(3, 500, 257, 72, dtype)
    d = w.clone()
    r = B.embedding_backward(dy, tokens, d_weight=d, scale=0.5, accumulate=True)
    assert r is d
    check_gradient(d, tokens, dy, 0.5, dtype, before=w)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shift,d", [(0, 64), (1, 64), (3, 61)])
def test_views_of_any_stride(shift, d, dtype):
    """Parts of larger buffers, off the 16-byte boundaries, replicas in turn row by row, tokens out of a wider table and one row
    of them for all replicas; nothing else of the buffers changes."""
    P, n, V = 3, 130, 90
    tokens, w, dy = inputs(P, n, V, d, dtype)
    dt = TYPES[dtype]

    def part(rows):
        whole = torch.full((rows, P, d + 16), 7.0, dtype=dt, device="cuda")
        return whole, whole[:, :, shift:shift + d].transpose(0, 1)
    _, ws = part(V)
    ws.copy_(w)
    buf_y, y = part(n)
    wide = torch.zeros((P, 2 * n + 1), dtype=tokens.dtype, device="cuda")
    ts = wide[:, 1::2]
    ts.copy_(tokens)
    assert B.embedding(ts, ws, out=y) is y
    check_forward(y, tokens, w, 1.0, dtype)
    buf_d, d_w = part(V)
    _, dys = part(n)
    dys.copy_(dy)
    B.embedding_backward(dys, ts, d_weight=d_w)
    check_gradient(d_w, tokens, dy, 1.0, dtype)
    for buf in (buf_y, buf_d):
        outside = torch.ones_like(buf, dtype=torch.bool)
        outside[:, :, shift:shift + d] = False
        assert (buf[outside] == 7.0).all()
    same = tokens[:1].expand(P, n)
    check_forward(B.embedding(same, w), same, w, 1.0, dtype)
    check_gradient(B.embedding_backward(dy, same, vocabulary=V), same, dy, 1.0, dtype)
    # one table for all replicas is read, never written
    check_forward(B.embedding(tokens, w[:1].expand(P, V, d)), tokens, w[:1].expand(P, V, d), 1.0, dtype)
    with pytest.raises(B.EventGradError):
        B.embedding_backward(dy, tokens, d_weight=w[:1].expand(P, V, d))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_what_stands_where_no_token_is_stays_there(dtype):
    """Infinities and NaN in rows that no token names, and in gradients of places without a token."""
    tokens, w, dy = inputs(2, 400, 500, 48, dtype)
    inside = (tokens >= 0) & (tokens < 500)
    named = torch.zeros(2, 500, dtype=torch.bool, device="cuda")
    for i in range(2):
        named[i, tokens[i][inside[i]]] = True
    w[~named] = float("nan")
    dy[~inside] = float("inf")
    y, d = B.embedding(tokens, w), B.embedding_backward(dy, tokens, vocabulary=500)
    assert torch.isfinite(y).all() and torch.isfinite(d).all()
    check_gradient(d, tokens, torch.where(inside[:, :, None], dy, torch.zeros_like(dy)), 1.0, dtype)


def test_no_places():
    empty = torch.zeros((2, 0), dtype=torch.int64, device="cuda")
    w = torch.randn((2, 30, 16), device="cuda")
    assert B.embedding(empty, w).shape == (2, 0, 16)
    d = w.clone()
    dy = torch.zeros((2, 0, 16), device="cuda")
    B.embedding_backward(dy, empty, d_weight=d, accumulate=True)
    assert torch.equal(d, w)
    B.embedding_backward(dy, empty, d_weight=d)
    assert (d == 0).all()


def test_gradient_against_differences():
    """Along random directions: the forward pass is linear in the table."""
    tokens, w, dy = inputs(2, 300, 200, 64, "fp32")
    d = B.embedding_backward(dy, tokens, vocabulary=200, scale=3.0).double()
    for seed in range(3):
        v = torch.randn(w.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        ahead, behind = (B.embedding(tokens, w + s * v, scale=3.0).double() for s in (0.5, -0.5))
        slope, by_hand = ((ahead - behind) * dy.double()).sum(), (d * v.double()).sum()
        # roundings of some 4e4 values of w + v/2 (2^-24 each, weights of size 3), random signs: below 1e-3
        assert abs(slope - by_hand) < 1e-2


def test_captured_and_replayed_with_other_tokens():
    tokens, w, dy = inputs(2, 600, 300, 64, "bf16")
    y, d = torch.empty_like(dy), torch.empty_like(w)

    def both():
        B.embedding(tokens, w, scale=2.0, out=y)
        B.embedding_backward(dy, tokens, scale=2.0, d_weight=d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (3, 4):
        t, w2, dy2 = inputs(2, 600, 300, 64, "bf16", seed=seed)
        tokens.copy_(t), w.copy_(w2), dy.copy_(dy2)
        graph.replay()
        check_forward(y, tokens, w, 2.0, "bf16")
        check_gradient(d, tokens, dy, 2.0, "bf16")


def test_two_streams_at_once():
    """Every call has a workspace of its own."""
    a, b = inputs(2, 3000, 700, 128, "fp32", seed=1), inputs(2, 3000, 700, 128, "fp32", seed=2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = [[], []]
    for _ in range(10):
        for s, (tokens, _, dy), out in zip(streams, (a, b), results):
            out.append(B.embedding_backward(dy, tokens, vocabulary=700, stream=s))
    torch.cuda.synchronize()
    for (tokens, _, dy), out in zip((a, b), results):
        check_gradient(out[0], tokens, dy, 1.0, "fp32")
        assert all(torch.equal(out[0], r) for r in out[1:])


def test_refusals():
    tokens, w, dy = inputs(2, 20, 30, 16, "fp32")
    for bad in (tokens.float(), tokens.short(), tokens[:1], tokens[0], tokens.cpu()):
        with pytest.raises(B.EventGradError):
            B.embedding(bad, w)
        with pytest.raises(B.EventGradError):
            B.embedding_backward(dy, bad, vocabulary=30)
    for bad in (w[0], w.double(), w.transpose(1, 2), w[:, :0]):
        with pytest.raises(B.EventGradError):
            B.embedding(tokens, bad)
    with pytest.raises(B.EventGradError):
        B.embedding(tokens, w, out=torch.empty_like(dy, dtype=torch.bfloat16))
    with pytest.raises(B.EventGradError):
        B.embedding(tokens, w, out=dy[:, :1].expand(2, 20, 16))
    with pytest.raises(B.EventGradError):
        B.embedding(tokens, w, scale=float("nan"))
    with pytest.raises(B.EventGradError, match="vocabulary"):
        B.embedding_backward(dy, tokens)
    with pytest.raises(B.EventGradError, match="accumulate"):
        B.embedding_backward(dy, tokens, vocabulary=30, accumulate=True)
    with pytest.raises(B.EventGradError):
        B.embedding_backward(dy, tokens, vocabulary=31, d_weight=w)
    with pytest.raises(B.EventGradError):
        B.embedding_backward(dy, tokens, vocabulary=0)
    with pytest.raises(B.EventGradError):
        B.embedding_backward(dy, tokens, d_weight=w.bfloat16())
    with pytest.raises(B.EventGradError, match="no_grad"):
        B.embedding(tokens, w.clone().requires_grad_())
    with pytest.raises(B.EventGradError, match="no_grad"):
        B.embedding_backward(dy.clone().requires_grad_(), tokens, vocabulary=30)
    with torch.no_grad():
        B.embedding(tokens, w.clone().requires_grad_())
