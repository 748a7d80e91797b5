"""The operators and the step together: a ring that trains a residual network of feed-forward blocks."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import residual_ffn_ring as R  # noqa: E402

pytestmark = pytest.mark.gpu


def reference_loss(net, params, x, target):
    """The network of the example in plain operations on 64-bit parameters ``[P, stride]``."""
    rms = lambda v: v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    vec = lambda t: net.view(params, t)[:, None]  # noqa: E731
    r = x.double()
    o = rms(r) * vec(0)
    for l in range(net.blocks):
        at = 1 + 7 * l
        wg, wu, wd = (net.view(params, at + q).transpose(1, 2) for q in range(3))
        y = (torch.nn.functional.silu(o @ wg) * (o @ wu)) @ wd
        r = vec(at + 5) * r + torch.sigmoid(vec(at + 4)) * (rms(y) * vec(at + 3))
        o = rms(r) * vec(at + 6)
    return o, (o - target.double()).pow(2).mean((1, 2)).sum()


@pytest.mark.parametrize("dtype,tolerance", [("fp32", 1e-5), ("bf16", 0.05)])
def test_gradients_of_the_whole_network(dtype, tolerance):
    """Against differentiation in 64 bits.  fp32: some ten operators in a row, each within a few 1e-7 of its result
    (1e-6 for a product); bf16: some fifteen roundings of 2^-8 / sqrt(3) in the mean on the longest way."""
    P, blocks, width, hidden, tokens = 3, 2, 48, 72, 33
    dt = R.TYPES[dtype]
    net = R.Network(P, blocks, width, hidden, dt)
    net.initialise(3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    net.params.add_(torch.randn(net.params.shape, generator=gen, device="cuda") * 0.05)    # replicas differ
    net.work.copy_(net.params)
    x, target = R.batch(P, tokens, width, 5, dt)
    out, kept = net.forward(x)
    net.backward(x, kept, ((out.float() - target) * (2.0 / (tokens * width))).to(dt))
    leaf = net.work.double().requires_grad_()
    want_out, loss = reference_loss(net, leaf, x, target)
    (want,) = torch.autograd.grad(loss, leaf)
    want_out = want_out.detach()
    assert float((out.double() - want_out).norm() / want_out.norm()) < tolerance
    for t in range(len(net.shapes)):
        got, ref = net.view(net.grads, t).double(), net.view(want, t)
        assert float((got - ref).norm()) <= tolerance * float(ref.norm()), t


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_training_lowers_the_loss_and_sends_fewer_messages(dtype):
    losses, sent = R.train(replicas=4, blocks=2, width=32, hidden=48, tokens=64, steps=40, dtype=dtype)
    assert losses[-1] < 0.7 * losses[0]
    assert 0.0 < sent < 1.0
