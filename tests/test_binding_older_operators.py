"""A build of the library that has the operators around the step, but none of those of a language model, goes on serving the former.
No compute call is made here (no GPU needed)."""
import os
import subprocess

import test_binding_without_operators as W
from paper_2103_07454_b200 import binding as B

LATER = {name for name in B.EXPORTS if name.startswith(("eg_embedding", "eg_head_norm", "eg_orthogonalise"))}

ASKS = """
import torch
from paper_2103_07454_b200 import binding as B
x, t = torch.zeros(1, 2, 8), torch.zeros(1, 2, dtype=torch.int64)
def says(call, text):
    try:
        call()
    except B.EventGradError as e:
        assert text in str(e), e
    else:
        raise AssertionError("a call on the host was taken")
w = torch.zeros(1, 8, 8)
for call in (lambda: B.residual_norm(x, x), lambda: B.feed_forward(x, w, w, w)):
    says(call, "no CUDA device")
for call in (lambda: B.embedding(t, w), lambda: B.embedding_backward(x, t, vocabulary=8), lambda: B.head_norm(x[None], None),
             lambda: B.head_norm_backward(x[None], None, x[None], None), lambda: B.orthogonalise([w])):
    says(call, "build")
print("done")
"""


def test_with_a_library_from_before_the_operators_of_a_language_model(tmp_path):
    assert len(LATER) == 8
    src = tmp_path / "older.c"
    src.write_text("\n".join(f"int {name}(void) {{ return 0; }}" for name in B.EXPORTS if name not in LATER))
    lib = tmp_path / "older.so"
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    W.run(ASKS, EG_LIBRARY=str(lib))
