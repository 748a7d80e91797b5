"""Adding to a table's gradient: by one launch for few places, by three for many, off the 16-byte boundaries too."""
import pytest
import torch

import test_gpu_embedding as E
from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(E.TYPES))
@pytest.mark.parametrize("P,n,V,d", [(1, 1, 1, 1), (4, 1, 1000, 64), (2, 31, 7, 33), (1, 200, 3, 40), (2, 256, 300, 96), (2, 257, 300, 96), (3, 777, 1009, 509),
                                     (1, 40000, 50, 24), (5, 333, 513, 1032)])
def test_adds_to_what_is_there(P, n, V, d, dtype):
    tokens, w, dy = E.inputs(P, n, V, d, dtype, seed=1, bits=32 if n % 2 else 64)
    got = w.clone()
    assert B.embedding_backward(dy, tokens, d_weight=got, scale=1.7, accumulate=True) is got
    E.check_gradient(got, tokens, dy, 1.7, dtype, before=w)


@pytest.mark.parametrize("n", [0, 40, 600])
def test_rows_of_no_token_keep_what_they_hold(n):
    """Infinities and NaN too."""
    tokens, w, dy = E.inputs(2, n, 90, 48, "bf16", seed=2)
    for i in range(2):
        tokens[i][tokens[i] == 17] = -1
    w[:, 17, :24], w[:, 17, 24:] = float("nan"), float("inf")
    got = w.clone()
    B.embedding_backward(dy, tokens, d_weight=got, accumulate=True)
    assert torch.equal(got[:, 17].view(torch.int16), w[:, 17].view(torch.int16))
    assert torch.isfinite(got[:, :17]).all() and torch.isfinite(got[:, 18:]).all()
