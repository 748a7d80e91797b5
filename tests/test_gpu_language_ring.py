"""The operators of a language model on the ring together: a block with attention trained on tokens, its gradients against
differentiation in 64 bits, its matrices' gradients made orthogonal, clipped and handed to the step."""
import math

import pytest
import torch

from paper_2103_07454_b200 import binding as B

pytestmark = pytest.mark.gpu

P, N, V, D, F, HQ, HK, DH = 3, 37, 53, 64, 96, 4, 2, 16
HEADS = HQ + 2 * HK
#: the tensors of a replica: table (also the output's matrix), norms, projection into heads and back, head norms, feed-forward block
SHAPES = dict(table=(V, D), pre=(D,), qkv=(HEADS * DH, D), w_q=(DH,), w_k=(DH,), out=(D, HQ * DH), mid=(D,), gate=(F, D), up=(F, D), down=(D, F),
              last=(D,))
MATRICES = ("qkv", "out", "gate", "up", "down")
SCALE = math.sqrt(D)


def views(ring, buffer):
    return {name: ring.view(buffer, t, shape) for t, (name, shape) in enumerate(SHAPES.items())}


def attention(q, k, v):
    """Causal, ``[P, rows, heads, width]``; several heads of queries share one of keys."""
    k, v = (x.repeat_interleave(HQ // HK, dim=2) for x in (k, v))
    s = torch.einsum("pnhd,pmhd->phnm", q, k) / math.sqrt(DH)
    s = s.masked_fill(torch.ones(N, N, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    return torch.einsum("phnm,pmhd->pnhd", torch.softmax(s, -1), v)


def loss_of(logits, targets):
    there = targets >= 0
    picked = torch.log_softmax(logits, -1).gather(-1, targets.clamp(min=0)[..., None])[..., 0]
    return -(picked * there).sum()


def reference(w, tokens, positions, targets):
    """The network in plain operations."""
    rms = lambda x: x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    col = lambda name: w[name][:, None]  # noqa: E731
    at = tokens.clamp(min=0)
    r = torch.stack([t[i] for t, i in zip(w["table"], at)]) * SCALE * (tokens >= 0)[..., None]
    heads = (rms(r) * col("pre") @ w["qkv"].mT).view(P, N, HEADS, DH)
    angle = positions.double()[..., None, None] * 10000.0 ** (-torch.arange(0, DH, 2, device="cuda").double() / DH)
    turned = []
    for x, name in ((heads[:, :, :HQ], "w_q"), (heads[:, :, HQ:HQ + HK], "w_k")):
        z = rms(x) * w[name][:, None, None]
        a, b = z[..., :DH // 2], z[..., DH // 2:]
        turned.append(torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1))
    r = r + attention(*turned, heads[:, :, HQ + HK:]).flatten(2) @ w["out"].mT
    o = rms(r) * col("mid")
    r = r + (torch.nn.functional.silu(o @ w["gate"].mT) * (o @ w["up"].mT)) @ w["down"].mT
    return loss_of(rms(r) * col("last") @ w["table"].mT, targets)


def gradients(ring, params, grads, tokens, positions, targets):
    """The same by the operators, with torch's attention, projections and loss between them; gradients go into ``grads``."""
    w, g = views(ring, params), views(ring, grads)
    x = B.embedding(tokens, w["table"], scale=SCALE)
    r0, o0 = B.residual_norm(None, x, w_pre=w["pre"])
    qkv = (o0 @ w["qkv"].mT).view(P, N, HEADS, DH)
    q, k, v = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HK], qkv[:, :, HQ + HK:]
    qr, kr = B.head_norm(q, k, w_q=w["w_q"], w_k=w["w_k"], positions=positions)
    with torch.enable_grad():
        leaves = [t.detach().requires_grad_() for t in (qr, kr, v)]
        mixed = attention(*leaves).flatten(2)
    y1 = mixed.detach() @ w["out"].mT
    r1, o1 = B.residual_norm(y1, r0, w_pre=w["mid"])
    y2, saved = B.feed_forward(o1, w["gate"], w["up"], w["down"], save=True)
    r2, o2 = B.residual_norm(y2, r1, w_pre=w["last"])
    with torch.enable_grad():
        logits = (o2 @ w["table"].mT).requires_grad_()
        loss = loss_of(logits, targets)
    (d_logits,) = torch.autograd.grad(loss, logits)

    # the output's matrix is the table: its gradient first, the embedding's added to it in the end
    torch.bmm(d_logits.mT, o2, out=g["table"])
    dy2, dr1, _ = B.residual_norm_backward(None, d_logits @ w["table"], y2, r1, w_pre=w["last"], d_weights=(None, None, None, g["last"]))
    do1, _ = B.feed_forward_backward(dy2, o1, w["gate"], w["up"], w["down"], saved, d_weights=(g["gate"], g["up"], g["down"]))
    dy1, dr0, _ = B.residual_norm_backward(dr1, do1, y1, r0, w_pre=w["mid"], d_weights=(None, None, None, g["mid"]))
    torch.bmm(dy1.mT, mixed.detach(), out=g["out"])
    d_qr, d_kr, d_v = torch.autograd.grad(mixed, leaves, dy1 @ w["out"])
    d_qkv = torch.empty_like(qkv)
    d_qkv[:, :, HQ + HK:] = d_v
    B.head_norm_backward(d_qr, d_kr, q, k, w_q=w["w_q"], w_k=w["w_k"], positions=positions, dq=d_qkv[:, :, :HQ], dk=d_qkv[:, :, HQ:HQ + HK],
                         d_weights=(g["w_q"], g["w_k"]))
    d_qkv = d_qkv.flatten(2)
    torch.bmm(d_qkv.mT, o0, out=g["qkv"])
    _, dx, _ = B.residual_norm_backward(dr0, d_qkv @ w["qkv"], None, x, w_pre=w["pre"], d_weights=(None, None, None, g["pre"]))
    B.embedding_backward(dx, tokens, scale=SCALE, d_weight=g["table"], accumulate=True)
    return loss.detach()


def start(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ring = B.EventGrad(P, [math.prod(s) for s in SHAPES.values()])
    params = ring.empty_params()
    params.zero_()
    for name, v in views(ring, params).items():
        noise = torch.randn(v.shape, generator=gen, device="cuda")
        v.copy_(1 + 0.1 * noise if v.dim() == 2 else noise * (0.1 if name == "table" else v.shape[2] ** -0.5))
    tokens = torch.randint(0, V, (P, N), generator=gen, device="cuda")
    tokens[1, 30:] = -1                                     # a shorter sequence
    targets = torch.where(tokens >= 0, (tokens + 1) % V, -1)
    positions = torch.arange(N, device="cuda").expand(P, N) + 1000
    return ring, params, tokens, positions, targets


@torch.no_grad()
def test_gradients_of_a_block_with_attention():
    """fp32 against 64 bits: some fifteen operators in a row, each within a few 1e-7 of its result (1e-6 for a product)."""
    ring, params, tokens, positions, targets = start(0)
    grads = ring.empty_params()
    grads.zero_()
    loss = gradients(ring, params, grads, tokens, positions, targets)
    with torch.enable_grad():
        leaf = params.double().requires_grad_()
        want_loss = reference(views(ring, leaf), tokens, positions, targets)
        (want,) = torch.autograd.grad(want_loss, leaf)
    assert abs(float(loss) - float(want_loss)) < 1e-5 * abs(float(want_loss))
    for name, got in views(ring, grads).items():
        ref = views(ring, want)[name]
        assert float((got.double() - ref).norm()) <= 2e-5 * float(ref.norm()), name
    ring.close()


@torch.no_grad()
def test_orthogonal_updates_reach_the_step():
    """Gradients, orthogonal updates of the matrices, clipping, step: three times; every update of a matrix is what the definition makes
    of its gradients so far, and the parameters move by it."""
    ring, params, tokens, positions, targets = start(1)
    grads, velocity = ring.empty_params(), ring.empty_params()
    grads.zero_(), velocity.zero_()
    so_far = {name: 0.0 for name in MATRICES}
    for _ in range(3):
        gradients(ring, params, grads, tokens, positions, targets)
        g, v = views(ring, grads), views(ring, velocity)
        raw = {name: g[name].clone().double() for name in MATRICES}
        B.orthogonalise([g[m] for m in MATRICES], velocity=[v[m] for m in MATRICES], momentum=0.9, scale=[0.2 * max(SHAPES[m]) ** 0.5 for m in MATRICES])
        for name in MATRICES:
            so_far[name] = 0.9 * so_far[name] + raw[name]
            x = raw[name] + 0.9 * so_far[name]
            x = x / x.pow(2).sum((1, 2), keepdim=True).sqrt()
            flip = x.shape[1] > x.shape[2]
            x = x.mT if flip else x
            for _ in range(5):
                a = x @ x.mT
                x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
            x = (x.mT if flip else x) * (0.2 * max(SHAPES[name]) ** 0.5)
            # few tokens: gradients of low rank, whose roundings grow 484 times in the directions without weight
            assert float((g[name].double() - x).norm()) < 3e-4 * float(x.norm()), name
        norms = ring.clip_gradients(grads, 1e9)
        assert torch.isfinite(norms).all()
        before = params.clone()
        ring.step(params, grads, 0.01)
        assert not torch.equal(params, before) and torch.isfinite(params).all()
    assert B.operator_status() == 0
    ring.close()
