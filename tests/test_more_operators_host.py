"""Host side of the operators of a language model on the ring: what is refused before anything reaches a device."""
import ctypes as C

import pytest
import torch

from paper_2103_07454_b200 import binding as B

INVALID = 1
A = 1 << 20                       # stands for an aligned device address; none of these calls gets as far as using it


class Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("replica_stride", C.c_int64), ("row_stride", C.c_int64)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("replica_stride", C.c_int64), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class Embedding(C.Structure):
    _fields_ = ([(n, C.c_int64) for n in ("P", "rows", "vocabulary", "width", "dtype", "token_bytes", "accumulate")] +
                [("scale", C.c_double), ("tokens", C.c_void_p), ("token_replica_stride", C.c_int64), ("token_stride", C.c_int64)] +
                [(n, Matrix) for n in ("weight", "out", "dy", "d_weight")])


class HeadNorm(C.Structure):
    _fields_ = ([(n, C.c_int64) for n in ("P", "rows", "q_heads", "k_heads", "width", "dtype", "rotary", "interleaved")] +
                [("base", C.c_double), ("eps", C.c_double), ("positions", C.c_void_p)] +
                [(n, C.c_int64) for n in ("position_bytes", "position_replica_stride", "position_stride")] +
                [(n, Matrix) for n in ("w_q", "w_k")] + [(n, Heads) for n in ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk")] +
                [(n, Matrix) for n in ("d_w_q", "d_w_k")])


def library():
    lib = B.load_library()
    for f in (lib.eg_embedding_workspace, lib.eg_head_norm_workspace):
        f.restype = C.c_int64
    for f in (lib.eg_embedding_backward, lib.eg_head_norm_backward):
        f.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    return lib


def embedding(**change):
    P, n, V, d = 2, 10, 30, 64
    v = dict(P=P, rows=n, vocabulary=V, width=d, dtype=B.BF16, token_bytes=8, accumulate=0, scale=1.0, tokens=A, token_replica_stride=n,
             token_stride=1, weight=Matrix(A, V * d, d), out=Matrix(A, n * d, d), dy=Matrix(A, n * d, d), d_weight=Matrix(A, V * d, d))
    v.update(change)
    return Embedding(**v)


BAD = [dict(P=0), dict(P=65536), dict(rows=-1), dict(vocabulary=0), dict(vocabulary=(1 << 30) + 1), dict(width=0), dict(width=(1 << 24) + 1),
       dict(dtype=3), dict(token_bytes=2), dict(tokens=None), dict(tokens=A + 4), dict(token_stride=-1), dict(token_replica_stride=-1),
       dict(scale=float("inf")), dict(scale=float("nan"))]


@pytest.mark.parametrize("bad", BAD)
def test_embedding_refuses(bad):
    lib = library()
    q = embedding(**bad)
    assert lib.eg_embedding(C.byref(q), None) == INVALID
    assert lib.eg_embedding_workspace(C.byref(q)) == 0
    assert lib.eg_embedding_backward(C.byref(q), A, 1 << 40, None) == INVALID


@pytest.mark.parametrize("bad", [Matrix(None, 640, 64), Matrix(A + 1, 640, 64), Matrix(A, 639, 64), Matrix(A, 640, 63), Matrix(A, 640, -64), Matrix(A, -1, 64),
                                 Matrix(A, 64, 127), Matrix(A, 0, 64), Matrix(A, 64, 0)])
def test_embedding_refuses_results_that_fall_on_one_another(bad):
    lib = library()
    assert lib.eg_embedding(C.byref(embedding(out=bad)), None) == INVALID
    q = embedding(vocabulary=10, d_weight=bad)
    assert lib.eg_embedding_backward(C.byref(q), A, 1 << 40, None) == INVALID and lib.eg_embedding_workspace(C.byref(q)) == 0


def test_embedding_refuses_missing_operands_and_small_workspaces():
    lib = library()
    assert lib.eg_embedding(C.byref(embedding(weight=Matrix())), None) == INVALID
    assert lib.eg_embedding_backward(C.byref(embedding(dy=Matrix())), A, 1 << 40, None) == INVALID
    q = embedding()
    need = lib.eg_embedding_workspace(C.byref(q))
    assert need >= 2 * 10 * 2 * 4
    for w, size in ((A, need - 1), (A + 8, need), (None, need)):
        assert lib.eg_embedding_backward(C.byref(q), w, size, None) == INVALID
    for good in (Matrix(A, 64, 128), Matrix(A, 700, 70), Matrix(A, 72, 136)):       # replicas in turn, room between
        assert lib.eg_embedding_workspace(C.byref(embedding(vocabulary=10, d_weight=good))) == need
    assert lib.eg_embedding(None, None) == INVALID and lib.eg_embedding_backward(None, A, 1 << 40, None) == INVALID


def head_norm(**change):
    P, n, hq, hk, d = 2, 10, 4, 2, 64
    v = dict(P=P, rows=n, q_heads=hq, k_heads=hk, width=d, dtype=B.BF16, rotary=64, interleaved=0, base=1e4, eps=1e-6, positions=A, position_bytes=8,
             position_replica_stride=n, position_stride=1, w_q=Matrix(A, d, 0), w_k=Matrix(A, d, 0), d_w_q=Matrix(A, d, 0), d_w_k=Matrix(A, d, 0))
    for name, h in (("q", hq), ("k", hk)):
        for form in (name, name + "_out", "d" + name + "_out", "d" + name):
            v[form] = Heads(A, n * h * d, h * d, d)
    v.update(change)
    return HeadNorm(**v)


@pytest.mark.parametrize("bad", [dict(P=0), dict(P=65536), dict(rows=-1), dict(q_heads=0), dict(q_heads=65536), dict(k_heads=-1), dict(width=0),
                                 dict(width=257), dict(dtype=3), dict(rotary=3), dict(rotary=-2), dict(rotary=66), dict(base=0.0), dict(base=float("nan")),
                                 dict(eps=-1e-9), dict(eps=float("nan")), dict(position_bytes=2), dict(positions=A + 4), dict(position_stride=-1),
                                 dict(w_q=Matrix(A + 1, 64, 0)), dict(w_k=Matrix(A, -1, 0)), dict(q=Heads()), dict(k=Heads()), dict(q=Heads(A + 1, 2560, 256, 64)),
                                 dict(q=Heads(A, 2560, 256, -64)), dict(k_heads=0)])
def test_head_norm_refuses(bad):
    lib = library()
    q = head_norm(**bad)
    assert lib.eg_head_norm(C.byref(q), None) == INVALID
    assert lib.eg_head_norm_backward(C.byref(q), A, 1 << 40, None) == INVALID


@pytest.mark.parametrize("bad", [Heads(A, 2560, 256, 63), Heads(A, 2559, 256, 64), Heads(A, 2560, 255, 64), Heads(A, 0, 256, 64), Heads(A, 2560, 0, 64),
                                 Heads(A, 2560, 256, 0), Heads(A, 64, 256, 64), Heads(A, 2560, 64, 639), Heads(A, 256, 511, 64)])
def test_head_norm_refuses_results_that_fall_on_one_another(bad):
    lib = library()
    assert lib.eg_head_norm(C.byref(head_norm(q_out=bad)), None) == INVALID
    assert lib.eg_head_norm_backward(C.byref(head_norm(dq=bad)), A, 1 << 40, None) == INVALID
    assert lib.eg_head_norm(C.byref(head_norm(q_out=Heads())), None) == INVALID


def test_head_norm_refuses_what_does_not_belong_together():
    lib = library()
    for bad in (dict(dq_out=Heads()), dict(dk_out=Heads()), dict(w_q=Matrix()), dict(d_w_q=Matrix(A, 63, 0))):
        assert lib.eg_head_norm_backward(C.byref(head_norm(**bad)), A, 1 << 40, None) == INVALID
    assert lib.eg_head_norm(None, None) == INVALID and lib.eg_head_norm_backward(None, A, 1 << 40, None) == INVALID


def test_tensors_on_the_host_are_refused():
    t, w, q = torch.zeros(1, 3, dtype=torch.int64), torch.zeros(1, 5, 8), torch.zeros(1, 3, 2, 8)
    with pytest.raises(B.EventGradError):
        B.embedding(t, w)
    with pytest.raises(B.EventGradError):
        B.embedding_backward(torch.zeros(1, 3, 8), t, vocabulary=5)
    with pytest.raises(B.EventGradError):
        B.head_norm(q, q)
    with pytest.raises(B.EventGradError):
        B.head_norm_backward(q, q, q, q)


class OrthogonalMatrix(C.Structure):
    _fields_ = [("rows", C.c_int64), ("columns", C.c_int64), ("scale", C.c_double)] + [(n, Matrix) for n in ("grad", "out", "velocity", "velocity_out")]


class Orthogonalise(C.Structure):
    _fields_ = ([(n, C.c_int64) for n in ("P", "count", "dtype", "out_dtype", "steps", "nesterov")] +
                [("momentum", C.c_double), ("coefficients", C.POINTER(C.c_double)), ("matrices", C.POINTER(OrthogonalMatrix))])


def orthogonalise(matrices=None, coefficients=None, **change):
    """One 64 x 96 matrix of 2 replicas with a velocity, unless others are given; `matrices`: changes of it, one each."""
    P, r, c = 2, 64, 96
    all_ = []
    for m in matrices or [{}]:
        v = dict(rows=r, columns=c, scale=1.0, grad=Matrix(A, r * c, c), out=Matrix(A, r * c, c), velocity=Matrix(A, r * c, c), velocity_out=Matrix())
        v.update(m)
        all_.append(OrthogonalMatrix(**v))
    q = dict(P=P, count=len(all_), dtype=B.BF16, out_dtype=B.BF16, steps=5, nesterov=1, momentum=0.95, matrices=(OrthogonalMatrix * len(all_))(*all_))
    if coefficients is not None:
        q["coefficients"] = (C.c_double * len(coefficients))(*coefficients)
    q.update(change)
    return Orthogonalise(**q)


def workspace(q):
    lib = library()
    lib.eg_orthogonalise_workspace.restype = C.c_int64
    return lib.eg_orthogonalise_workspace(C.byref(q))


def refused(q):
    lib = library()
    lib.eg_orthogonalise.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    return workspace(q) == 0 and lib.eg_orthogonalise(C.byref(q), A, 1 << 50, None) == INVALID


@pytest.mark.parametrize("bad", [dict(P=0), dict(P=4097), dict(count=-1), dict(dtype=3), dict(out_dtype=3), dict(out_dtype=B.F16), dict(dtype=B.F32), dict(steps=0),
                                 dict(steps=65), dict(momentum=float("nan")), dict(momentum=float("inf")), dict(matrices=[dict(rows=0)]),
                                 dict(matrices=[dict(columns=(1 << 20) + 1)]), dict(matrices=[dict(scale=float("nan"))]), dict(matrices=[dict(grad=Matrix())]),
                                 dict(matrices=[dict(out=Matrix())]), dict(matrices=[dict(out=Matrix(A, 6143, 96))]), dict(matrices=[dict(out=Matrix(A, 6144, 95))]),
                                 dict(matrices=[dict(out=Matrix(A, 0, 96))]), dict(matrices=[dict(grad=Matrix(A + 1, 6144, 96))]),
                                 dict(matrices=[dict(velocity=Matrix(A + 2, 6144, 96))]), dict(matrices=[dict(velocity=Matrix(A, 6143, 96))]),
                                 dict(matrices=[dict(velocity=Matrix(), velocity_out=Matrix(A, 6144, 96))]), dict(matrices=[{}, dict(rows=-1)]),
                                 dict(coefficients=[float("nan")] * 15), dict(coefficients=[2e4, 0.0, 0.0] * 5), dict(coefficients=[3.0, 0.0, 0.0] * 5)])
def test_orthogonalise_refuses(bad):
    assert refused(orthogonalise(**bad))


def test_orthogonalise_takes_what_it_should():
    lib = library()
    one = workspace(orthogonalise())
    assert one >= 2 * (3 * 2 + 2) * 8192                      # of two replicas: X twice and its lower parts, A and B
    assert workspace(orthogonalise(out_dtype=B.F32)) >= one
    assert workspace(orthogonalise(matrices=[{}] * 3)) > one
    assert workspace(orthogonalise(coefficients=[1.5, -0.5, 0.0] * 5)) == one
    assert workspace(orthogonalise(coefficients=[1.875, -1.25, 0.375] * 64, steps=64)) == one
    assert workspace(orthogonalise(matrices=[dict(out=Matrix(A, 96, 192), grad=Matrix(A, 0, 0))])) == one
    assert workspace(orthogonalise(matrices=[dict(velocity=Matrix(A, 0, 96), velocity_out=Matrix(A, 6144, 96))])) == one
    big = [dict(rows=8192, columns=16384, grad=Matrix(A, 1 << 27, 16384), out=Matrix(A, 1 << 27, 16384), velocity=Matrix())]
    assert workspace(orthogonalise(matrices=big * 3)) < 2 * workspace(orthogonalise(matrices=big))   # one after another
    q = orthogonalise()
    lib.eg_orthogonalise.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
    for w, size in ((A, one - 1), (A + 64, one), (None, one)):
        assert lib.eg_orthogonalise(C.byref(q), w, size, None) == INVALID
    assert lib.eg_orthogonalise(C.byref(orthogonalise(count=0)), None, 0, None) == 0
    assert lib.eg_orthogonalise(None, A, one, None) == INVALID


def test_matrices_on_the_host_are_refused():
    with pytest.raises(B.EventGradError):
        B.orthogonalise([torch.zeros(1, 4, 8)])
