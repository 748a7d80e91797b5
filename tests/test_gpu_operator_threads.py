"""Operators called by several threads at once, each with its own stream, for the first time in a process: what they look up once per
device is looked up by all of them."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import threading
import torch
from paper_2103_07454_b200 import binding as B

def inputs(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    return dict(x=normal(2, 90, 64), gate=normal(2, 96, 64), up=normal(2, 96, 64), down=normal(2, 64, 96), heads=normal(2, 90, 4, 32), table=normal(2, 50, 64),
                tokens=torch.randint(-1, 50, (2, 90), generator=gen, device="cuda"), matrix=normal(2, 70, 130))

def all_of_them(t):
    y, saved = B.feed_forward(t["x"], t["gate"], t["up"], t["down"], save=True)
    dx, dw = B.feed_forward_backward(t["x"], t["x"], t["gate"], t["up"], t["down"], saved)
    r = B.residual_norm(t["x"], t["x"], w_pre=t["x"][:, 0])
    e = B.embedding(t["tokens"], t["table"])
    d = B.embedding_backward(e, t["tokens"], vocabulary=50)
    q, _ = B.head_norm(t["heads"], None, w_q=t["heads"][:, 0, 0])
    o = [torch.empty_like(t["matrix"]), torch.empty(t["matrix"].shape, device="cuda")]
    for out in o:
        B.orthogonalise([t["matrix"]], out=[out])
    return [y, dx, *dw, *r, e, d, q, *o]

sets = [inputs(seed) for seed in range(4)]
torch.cuda.synchronize()
start, results, failed = threading.Barrier(4), [None] * 4, []

def work(k):
    try:
        with torch.cuda.stream(torch.cuda.Stream()):
            start.wait(60)
            for _ in range(20):
                results[k] = all_of_them(sets[k])
            torch.cuda.current_stream().synchronize()
    except BaseException as e:
        failed.append(repr(e))

threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
[t.start() for t in threads]
[t.join(120) for t in threads]
assert not failed and not any(t.is_alive() for t in threads), failed
for t, got in zip(sets, results):
    for a, b in zip(got, all_of_them(t)):
        assert torch.equal(a, b)
assert B.operator_status() == 0
print("done")
"""


def test_first_calls_of_several_threads():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), r.stderr
