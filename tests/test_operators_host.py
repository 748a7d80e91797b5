"""Host side of the operators around the step: what is refused before anything reaches a device, and sizes."""
import struct

import pytest
import torch

from paper_2103_07454_b200 import binding as B

INVALID = 1
A = 1 << 20                       # stands for an aligned device address; none of these calls gets as far as using it


def norm_args(P=2, rows=4, width=64, dtype=B.F32, eps=1e-6, workspace=(A, 1 << 30), **mats):
    names = ("y", "residual", "w_post", "gate", "scale", "w_pre", "residual_out", "out", "d_residual_out", "d_out", "dy", "d_residual",
             "d_w_post", "d_gate", "d_scale", "d_w_pre")
    full = {n: (A, rows * width, width) for n in names}
    full.update(mats)
    return B._NORM_ARGS.pack(P, rows, width, dtype, eps, *(v for n in names for v in (full[n] or (0, 0, 0))), *workspace)


@pytest.mark.parametrize("bad", [dict(P=0), dict(P=70000), dict(rows=-1), dict(width=0), dict(width=8193), dict(dtype=3), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(residual=None), dict(y=None), dict(y=(A + 2, 256, 64)),
                                 dict(residual_out=(A, 256, 63)), dict(out=(A, 10, 64)), dict(y=(A, 256, -64))])
def test_norm_refuses(bad):
    lib = B.load_library()
    assert lib.eg_residual_norm(norm_args(**bad), None) == INVALID
    if bad.keys() <= {"P", "rows", "width", "dtype", "eps", "residual", "y"}:
        assert lib.eg_residual_norm_backward(norm_args(**bad), None) == INVALID


def test_norm_refuses_what_does_not_belong_together():
    lib = B.load_library()
    none = dict(w_post=None, gate=None)
    assert lib.eg_residual_norm(norm_args(w_pre=None), None) == INVALID                     # out without w_pre
    assert lib.eg_residual_norm(norm_args(out=None), None) == INVALID                       # w_pre without out
    assert lib.eg_residual_norm(norm_args(residual_out=None), None) == INVALID              # y without a place for r'
    assert lib.eg_residual_norm(norm_args(y=None, w_pre=None, out=None, residual_out=None, **none), None) == INVALID
    assert lib.eg_residual_norm_backward(norm_args(w_pre=None), None) == INVALID            # d_out without w_pre
    assert lib.eg_residual_norm_backward(norm_args(y=None, **none), None) == INVALID        # dy without y
    assert lib.eg_residual_norm_backward(norm_args(scale=None), None) == INVALID            # d_scale without scale
    assert lib.eg_residual_norm_backward(norm_args(d_gate=(A, 63, 0)), None) == INVALID     # replicas on one another
    need = lib.eg_residual_norm_workspace(2, 64)
    assert need > 0
    assert lib.eg_residual_norm_backward(norm_args(workspace=(A, need - 1)), None) == INVALID
    assert lib.eg_residual_norm_backward(norm_args(workspace=(A + 8, need)), None) == INVALID
    assert lib.eg_residual_norm_backward(norm_args(workspace=(0, need)), None) == INVALID


def ffn_args(P=2, rows=100, d=64, f=128, dtype=B.BF16, act=0, saved=(A, 1 << 40), **mats):
    shapes = dict(x=(rows, d), w_gate=(f, d), w_up=(f, d), w_down=(d, f), y=(rows, d), dy=(rows, d), dx=(rows, d), d_gate=(f, d),
                  d_up=(f, d), d_down=(d, f))
    full = {n: (A, r * c, c) for n, (r, c) in shapes.items()}
    full.update(mats)
    return B._FFN_ARGS.pack(P, rows, d, f, dtype, act, *(v for n in shapes for v in (full[n] or (0, 0, 0))), *saved)


@pytest.mark.parametrize("bad", [dict(P=0), dict(rows=-1), dict(d=0), dict(f=0), dict(d=(1 << 24) + 1), dict(dtype=3), dict(act=3), dict(x=None),
                                 dict(w_up=None), dict(w_down=(A + 1, 8192, 128)), dict(w_gate=(A, 8192, 63)), dict(x=(A, 6399, 64))])
def test_feed_forward_refuses(bad):
    lib = B.load_library()
    args = ffn_args(**bad)
    for backward, call in ((0, lib.eg_feed_forward), (1, lib.eg_feed_forward_backward)):
        assert lib.eg_feed_forward_workspace(args, backward) == 0
        assert call(args, A, 1 << 40, None) == INVALID


def test_feed_forward_refuses_missing_results_and_small_buffers():
    lib = B.load_library()
    assert lib.eg_feed_forward(ffn_args(y=None), A, 1 << 40, None) == INVALID
    assert lib.eg_feed_forward_backward(ffn_args(dy=None), A, 1 << 40, None) == INVALID
    assert lib.eg_feed_forward_backward(ffn_args(dx=(A, 6399, 64)), A, 1 << 40, None) == INVALID
    args = ffn_args()
    saved = lib.eg_feed_forward_saved_bytes(args)
    assert saved == 3 * 2 * 100 * 128 * 2
    for call, backward in ((lib.eg_feed_forward, 0), (lib.eg_feed_forward_backward, 1)):
        assert call(ffn_args(saved=(A, saved - 1)), A, 1 << 40, None) == INVALID
        assert call(ffn_args(saved=(A + 8, saved)), A, 1 << 40, None) == INVALID
    assert lib.eg_feed_forward_backward(ffn_args(saved=(0, 0)), A, 1 << 40, None) == INVALID
    need = lib.eg_feed_forward_workspace(args, 1)
    assert need >= 2 * 2 * 100 * 128 * 2                          # dG and dU
    assert lib.eg_feed_forward_backward(args, A, need - 1, None) == INVALID
    assert lib.eg_feed_forward_backward(args, 0, need, None) == INVALID


def test_workspace_follows_alignment_and_type():
    """Rows that cannot be read in place are copied, fp32 always (as three 16-bit parts)."""
    lib = B.load_library()
    in_place = lib.eg_feed_forward_workspace(ffn_args(), 0)
    assert in_place == 0                                          # H lies in `saved`
    assert lib.eg_feed_forward_workspace(ffn_args(saved=(0, 0)), 0) >= 2 * 100 * 128 * 2
    copied = lib.eg_feed_forward_workspace(ffn_args(x=(A + 2, 6400, 64)), 0)
    assert copied >= 2 * 100 * 64 * 2
    fp32 = lib.eg_feed_forward_workspace(ffn_args(dtype=B.F32), 0)
    assert fp32 >= 3 * 2 * 2 * (100 * 64 + 3 * 64 * 128)
    assert lib.eg_feed_forward_saved_bytes(ffn_args(dtype=B.F32)) == 2 * 100 * 128 * (4 + 4 + 6)


def test_clipping_needs_a_context():
    lib = B.load_library()
    assert lib.eg_clip_gradients(None, A, B.F32, 1.0, 0, A, A, None) == INVALID


def test_argument_records_have_the_headers_size():
    """eg_residual_norm_args: four integers, eps, sixteen matrices, workspace; eg_feed_forward_args: six integers, ten
    matrices, saved."""
    assert B._NORM_ARGS.size == 8 * (4 + 1 + 16 * 3 + 2)
    assert B._FFN_ARGS.size == 8 * (6 + 10 * 3 + 2)
    assert struct.calcsize("P") == 8


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(1, 2, 8)
    w = torch.zeros(1, 8, 8)
    with pytest.raises(B.EventGradError):
        B.feed_forward(x, w, w, w)
    with pytest.raises(B.EventGradError):
        B.residual_norm(x, x)
    with pytest.raises(B.EventGradError):
        B.residual_norm_backward(x, None, x, x)
    with pytest.raises(B.EventGradError):
        B.feed_forward_backward(x, x, w, w, w, torch.zeros(8, dtype=torch.uint8))


def test_feed_forward_takes_replicas_row_by_row():
    """[rows][P][columns], with room between; one element less and they overlap."""
    lib = B.load_library()
    need = lib.eg_feed_forward_workspace(ffn_args(saved=(0, 0)), 0)
    for x in ((A, 64, 128), (A, 64, 192), (A, 72, 136)):
        assert lib.eg_feed_forward_workspace(ffn_args(saved=(0, 0), x=x), 0) == need
    assert lib.eg_feed_forward_workspace(ffn_args(saved=(0, 0), x=(A + 2, 64, 128)), 0) > need
    for x in ((A, 63, 128), (A, 64, 127), (A, 0, 64), (A, 0, 1 << 20)):
        assert lib.eg_feed_forward_workspace(ffn_args(saved=(0, 0), x=x), 0) == 0
        assert lib.eg_feed_forward(ffn_args(x=x), A, 1 << 40, None) == INVALID


@pytest.mark.parametrize("rows,P", [(2, 2), (4, 2), (4, 3), (5, 2)])
def test_norm_refuses_results_that_fall_on_one_another(rows, P):
    """Replicas apart: at least (rows - 1) * row + width; in turn: a row of at least (P - 1) * replica + width."""
    lib = B.load_library()
    w = 64
    outs = ("residual_out", "out")
    grads = ("dy", "d_residual")
    for rep, row in (((rows - 1) * w + w - 1, w), (w, w * P - 1), (w, w), (3 * w * (rows - 1) + w - 1, 3 * w), (2 * w, 2 * w * (P - 1) + w - 1)):
        for name in outs + grads:
            call = lib.eg_residual_norm if name in outs else lib.eg_residual_norm_backward
            assert call(norm_args(P=P, rows=rows, width=w, **{name: (A, rep, row)}), None) == INVALID, (name, rep, row)
