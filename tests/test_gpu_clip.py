"""The gradient norm of a replica over its tensors, and clipping, against the formula in 64 bits."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# The norm is an fp64 sum rounded once to fp32 (2^-24); a result has the roundings of the factor
# and of the product (2^-24 each).  1.3e-7 > 2^-23.
RTOL = 1.3e-7
SETS = {
    "one": [1],
    "tiny": [3, 1, 5, 32, 33],
    "ragged": [4095, 4096, 4097, 7, 10000, 1],
    "many": [64] * 700 + [36864, 10],
}


def make(numel, P, dtype, seed=0, scale=1.0, padding=float("nan")):
    """(context, gradients in its layout with `padding` between the tensors, mask of the elements)"""
    eg = B.EventGrad(P, numel)
    mask = torch.zeros((P, eg.replica_stride), dtype=torch.bool, device="cuda")
    for o, n in zip(eg.tensor_offset, numel):
        mask[:, o:o + n] = True
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g = torch.randn((P, eg.replica_stride), generator=gen, device="cuda") * scale
    g = (g * torch.arange(1, P + 1, device="cuda")[:, None]).to(TYPES[dtype])
    return eg, torch.where(mask, g, torch.full_like(g, padding)), mask


def expected(g, mask, max_norm, zero_nonfinite=False):
    d = torch.where(mask, g.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    norm = d.pow(2).sum(1).sqrt()
    c = torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm))
    c = torch.where(norm.isnan(), norm, c)
    out = d * c[:, None]
    if zero_nonfinite:
        out[~norm.isfinite()] = 0.0
    return norm, out


def same(got, want, mask):
    got, want = got[mask].double(), want[mask]
    assert torch.equal(got.isnan(), want.isnan())
    ok = ~want.isnan()
    assert torch.all((got[ok] - want[ok]).abs() <= RTOL * want[ok].abs() + 1.5e-45)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("P", [1, 3, 16])
def test_norm_and_clipped_gradients(name, P, dtype):
    numel = SETS[name]
    eg, g, mask = make(numel, P, dtype)
    max_norm = 1.7 * math.sqrt(sum(numel))         # the first replica stays as it is, the others do not
    out = torch.full((P, eg.replica_stride), 7.0, device="cuda")
    norms = eg.clip_gradients(g, max_norm, out=out)
    want_n, want = expected(g, mask, max_norm)
    assert torch.all((norms.double() - want_n).abs() <= 6e-8 * want_n)
    same(out, want, mask)
    assert torch.all(out[~mask] == 7.0), "padding was written"
    again = torch.empty_like(out)
    assert torch.equal(eg.clip_gradients(g, max_norm, out=again), norms)
    assert torch.equal(again[mask], out[mask])


def test_in_place_and_default():
    eg, g, mask = make(SETS["ragged"], 3, "fp32", padding=5.0)
    want_n, want = expected(g, mask, 2.0)
    norms = eg.clip_gradients(g, 2.0)
    assert torch.all((norms.double() - want_n).abs() <= 6e-8 * want_n)
    same(g, want, mask)
    assert torch.all(g[~mask] == 5.0)


def test_more_replicas_than_blocks_meet_few_tiles():
    eg, g, mask = make([5], 1024, "bf16")
    out = torch.zeros(g.shape, device="cuda")
    norms = eg.clip_gradients(g, 1.0, out=out)
    want_n, want = expected(g, mask, 1.0)
    assert torch.all((norms.double() - want_n).abs() <= 6e-8 * want_n)
    same(out, want, mask)


def test_zero_norm_bound_zero_and_infinite_bound():
    eg, g, mask = make([40, 3], 2, "fp32")
    g[0] = 0.0
    out = torch.empty_like(g)
    assert eg.clip_gradients(g, 0.0, out=out)[0] == 0
    assert torch.all(out[mask] == 0)
    eg.clip_gradients(g, math.inf, out=out)
    assert torch.equal(out[mask], g[mask])


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_squares_beyond_the_range_of_32_bits(scale):
    eg, g, mask = make([500, 41], 2, "fp32", scale=scale)
    out = torch.empty_like(g)
    for max_norm in (scale, 1e-9):
        norms = eg.clip_gradients(g, max_norm, out=out)
        want_n, want = expected(g, mask, max_norm)
        assert torch.all((norms.double() - want_n).abs() <= 6e-8 * want_n)
        same(out, want, mask)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_replica_that_is_not_finite(value, zero, dtype):
    eg, g, mask = make(SETS["ragged"], 3, dtype)
    g[1, eg.tensor_offset[4] + 9] = value
    out = torch.empty(g.shape, device="cuda")
    norms = eg.clip_gradients(g, 1.0, out=out, zero_nonfinite=zero)
    _, want = expected(g, mask, 1.0, zero)
    assert not torch.isfinite(norms[1]) and torch.isfinite(norms[[0, 2]]).all()
    same(out, want, mask)


def test_on_another_stream_and_in_a_graph():
    eg, g, mask = make(SETS["ragged"], 4, "bf16")
    out = torch.zeros(g.shape, device="cuda")
    norms = torch.empty(4, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eg.clip_gradients(g, 1.0, out=out, norms=norms, stream=side)
    side.synchronize()
    want_n, want = expected(g, mask, 1.0)
    same(out, want, mask)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eg.clip_gradients(g, 1.0, out=out, norms=norms)
    g.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    _, want = expected(g, mask, 1.0)
    same(out, want, mask)
    assert torch.all((norms.double() - 2 * want_n).abs() <= 1.2e-7 * want_n)


def test_another_stream_while_the_first_is_busy_is_refused():
    eg, g, _ = make([1000], 2, "fp32", padding=0.0)
    eg.clip_gradients(g, 1.0)
    torch.cuda.synchronize()
    busy, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(50_000_000)
        eg.clip_gradients(g, 1.0)
    with pytest.raises(B.EventGradError, match="not allowed in this state"):
        eg.clip_gradients(g, 1.0, stream=other)
    torch.cuda.synchronize()
    eg.clip_gradients(g, 1.0, stream=other)
    torch.cuda.synchronize()


def test_refusals():
    eg, g, _ = make([1000, 3], 2, "fp32", padding=0.0)
    lib, p, s = eg._lib, g.data_ptr(), torch.cuda.current_stream().cuda_stream
    norms = torch.empty(2, device="cuda")
    n = norms.data_ptr()

    def call(grads=p, dtype=B.F32, max_norm=1.0, flags=0, out=p, norms=n, h=eg._h):
        return lib.eg_clip_gradients(h, grads, dtype, max_norm, flags, out, norms, s)

    assert call() == 0
    for kw in (dict(h=None), dict(grads=None), dict(out=None), dict(norms=None), dict(dtype=3), dict(dtype=-1),
               dict(max_norm=-1.0), dict(max_norm=math.nan), dict(flags=2), dict(grads=p + 4, out=p + 4),
               dict(dtype=B.BF16), dict(out=p + 16)):
        assert call(**kw) == 1, kw
    with pytest.raises(AssertionError):
        eg.clip_gradients(g.bfloat16(), 1.0)              # 16-bit gradients need an fp32 output
    with pytest.raises(AssertionError):
        eg.clip_gradients(g[:, :-32], 1.0)
    torch.cuda.synchronize()
