"""What the operators' kernels do around their bounded waits, by kernels of the test's own (operator_waits.cu) that use the same
device functions."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2103_07454_b200 import binding as B
from paper_2103_07454_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    to = str(tmp_path_factory.mktemp("kernels") / "operator_waits.so")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "operator_waits.cu")
    subprocess.run([build.NVCC, *build.FLAGS, "-shared", "-o", to, source], check=True)
    return C.CDLL(to)


def test_warps_that_meet_leave_a_walk_together(kernels):
    """Whichever of the two raises the flag, and whenever: both have walked as many turns, and none stays behind."""
    blocks = 61 * 64
    turns = torch.full((blocks, 2), -1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert kernels.walk(C.c_void_p(turns.data_ptr()), blocks, 1000, C.c_void_p(stream)) == 0
    turns = turns.cpu()
    assert torch.equal(turns[:, 0], turns[:, 1])
    raised = torch.arange(blocks) % 61
    # seen at the start of the next turn: a turn's meeting lies between the raising and the look
    assert torch.equal(turns[:, 0], (raised + 1).int())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_limits_of_waits_start_where_the_kernel_before_has_ended(kernels, dtype):
    """A predecessor that lets its successors start at once and then takes longer (1.6 s) than any wait may (about a second)."""
    g = torch.randn((2, 90, 200), generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").to(dtype)
    want, got = torch.empty_like(g), torch.empty_like(g)
    B.orthogonalise([g], out=[want])
    assert B.operator_status() == 0
    assert kernels.slow(C.c_uint64(1600000000), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    B.orthogonalise([g], out=[got])
    assert B.operator_status() == 0
    assert torch.equal(got, want)
