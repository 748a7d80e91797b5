"""The operators at sizes where another kernel, tile or run of rows takes over, against the formulas in 64 bits."""
import pytest
import torch

import test_gpu_feed_forward as F
import test_gpu_residual_norm as N
from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("P,n,d", [(2, 300, 4097), (1, 400, 8192), (3, 150, 5000), (2, 260, 6001), (4, 100, 2048), (3, 211, 1001), (9, 131, 77)])
def test_norm_streamed(P, n, d, dtype):
    x, w = N.inputs(P, n, d, dtype, seed=11)
    N.run_and_check(x, w, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(5, 50, 300), (7, 40, 1001), (37, 8, 64), (3, 49, 4100), (3, 90, 2001), (148, 2, 33), (1, 149, 520), (1, 148, 8191)])
def test_norm_short_runs(P, n, d, dtype):
    """One or two rows a CTA, runs that end with their replica and runs that do not."""
    x, w = N.inputs(P, n, d, dtype, seed=12)
    N.run_and_check(x, w, dtype)


@pytest.mark.parametrize("given", [(), ("w_pre",), ("w_post",), ("gate",), ("scale",), ("w_post", "w_pre"), ("gate", "w_pre")])
@pytest.mark.parametrize("d", [96, 333])
def test_norm_streamed_what_is_not_given_drops_out(given, d):
    x, w = N.inputs(2, 700, d, "fp32", seed=13, given=given)
    N.run_and_check(x, w, "fp32")


@pytest.mark.parametrize("n,d", [(700, 96), (700, 333), (200, 4104), (60, 96), (60, 333)])
def test_norm_rows_that_are_not_numbers_stay_alone(n, d):
    x, w = N.inputs(2, n, d, "fp32", seed=14)
    clean = (*B.residual_norm(x["y"], x["residual"], **w), *B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)[:2])
    x["y"][0, 3, 5] = float("nan")
    x["residual"][1, n - 1, d - 1] = float("inf")
    got = (*B.residual_norm(x["y"], x["residual"], **w), *B.residual_norm_backward(x["d_r"], x["d_o"], x["y"], x["residual"], **w)[:2])
    others = torch.ones(2, n, dtype=torch.bool, device="cuda")
    others[0, 3] = others[1, n - 1] = False
    for a, b in zip(got, clean):
        assert torch.all((a[others] - b[others]).abs() <= 2e-6 * b[others].abs().amax(-1, keepdim=True))
        assert not torch.isfinite(a[~others]).all()


@pytest.mark.parametrize("n", [9, 16, 17, 33, 64, 65])
@pytest.mark.parametrize("d,f", [(40, 72), (129, 257)])
def test_few_tokens_in_groups_fp32(n, d, f):
    t = F.inputs(2, n, d, f, "fp32", seed=n)
    F.check(dict(y=B.feed_forward(t["x"], t["w_gate"], t["w_up"], t["w_down"])), F.exact(t, "silu"), "fp32", ("y",))


@pytest.mark.parametrize("n", [3, 4, 5, 8, 16])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,f", [(41, 73), (129, 257), (64, 131)])
def test_few_tokens_in_groups_16_bit(n, d, f, dtype):
    t = F.inputs(3, n, d, f, dtype, seed=n)
    F.check(dict(y=B.feed_forward(t["x"], t["w_gate"], t["w_up"], t["w_down"])), F.exact(t, "silu"), dtype, ("y",))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("P,n,d,f", [(1, 20, 512, 1001), (2, 300, 1001, 512), (1, 4, 1032, 2600), (3, 5, 333, 1301), (2, 300, 296, 520), (1, 100, 200, 1500),
                                     (1, 1500, 88, 200), (1, 290, 520, 2056)])
def test_results_with_and_without_aligned_rows(P, n, d, f, dtype):
    """Rows of the results on 16-byte boundaries and off them, in one launch; few long tiles beside many short ones."""
    F.run_and_check(F.inputs(P, n, d, f, dtype, seed=15), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("spread", [1, 2, 3, 5])
def test_gradients_in_rows_of_any_stride(dtype, spread):
    """Nothing between the rows of a gradient is written."""
    P, n, d, f = 2, 40, 270, 330
    t = F.inputs(P, n, d, f, dtype, seed=16)
    flat = [torch.full((P, r, c + spread), 3.0, dtype=F.TYPES[dtype], device="cuda") for r, c in ((f, d), (f, d), (d, f))]
    got = F.run(t, "silu", d_weights=[m[:, :, 1:c + 1] if spread > 1 else m[:, :, :c] for m, c in zip(flat, (d, d, f))])
    F.check(got, F.exact(t, "silu"), dtype)
    for m, c in zip(flat, (d, d, f)):
        assert torch.all(m[:, :, c + (spread > 1):] == 3.0) and (spread == 1 or torch.all(m[:, :, 0] == 3.0))


def test_native_marshalling_refuses():
    """Wrong kinds of arguments are errors of the library, not of the interpreter."""
    x, w = N.inputs(1, 4, 64, "fp32")
    with pytest.raises(B.EventGradError):
        B.residual_norm(x["y"], 3.0)
    with pytest.raises(B.EventGradError):
        B.residual_norm(x["y"], x["residual"], w_post="w")
    with pytest.raises(B.EventGradError):
        B.residual_norm(x["y"], x["residual"], eps="a")
    with pytest.raises(B.EventGradError):
        B.feed_forward(x["y"], x["y"], None, x["y"])
    with pytest.raises(B.EventGradError):
        B.feed_forward_backward(x["y"], x["y"], x["y"], x["y"], x["y"], None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("P,n,d", [(2, 100, 4096), (1, 200, 4090), (1, 296, 4095), (1, 150, 3400)])
def test_norm_short_runs_of_the_widest_rows(P, n, d, dtype):
    """Column sums of nearly 48 KB in shared memory."""
    x, w = N.inputs(P, n, d, dtype, seed=17)
    N.run_and_check(x, w, dtype)
