"""The embedding's checks at the ends of what sizes and strides may be, before anything reaches a device."""
import ctypes as C

import pytest

from test_more_operators_host import A, INVALID, Matrix, embedding, library


@pytest.mark.parametrize("rows", [1 << 30, (1 << 29) + 1, 1 << 28])
@pytest.mark.parametrize("row", [1 << 34, (1 << 35) + 64, (1 << 36) - 1])
def test_replicas_that_fall_on_one_another_far_apart(rows, row):
    """What a replica spans passes 64 bits."""
    lib = library()
    for rep, good in ((63, False), (64, True), (row - 63, False), (0, False)):
        q = embedding(vocabulary=rows, d_weight=Matrix(A, rep, row))
        assert (lib.eg_embedding_workspace(C.byref(q)) > 0) == good, rep
        if not good:
            assert lib.eg_embedding_backward(C.byref(q), A, 1 << 62, None) == INVALID
