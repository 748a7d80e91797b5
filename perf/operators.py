"""The operators around a training step of a ring of replicas, as cases that can be timed and checked.

P replicas, each with weights of its own, train a residual network of gated feed-forward blocks; their
gradients are clipped and handed to the event-triggered step.  Three operators do that next to the step:

* ``feed_forward``    y = (act(x Wg^T) * (x Wu^T)) Wd^T of every replica, and its gradients;
* ``residual_norm``   r' = scale * r + sigmoid(gate) * rms(y) * w_post,  o = rms(r') * w_pre, and its gradients;
* ``clip``            the norm over all tensors of a replica, and the gradients scaled down to ``max_norm``.

Weights are views into one ``[P, stride]`` buffer, tensor after tensor, each on a 128-byte boundary of the
fp32 parameters: the layout that the step works on.  ``own`` False computes the operators in their plain form.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the gradients of the small 784-64-32-10 perceptron on 4 replicas: a call bound by its latency
        dict(name="clip_mlp_p4", op="clip", P=4, net="mlp", width=64, depth=1, dtype="fp32", share=0.5),
        # the ResNet-18 of 11.2 M parameters on 16 replicas, the size that the step itself is measured at
        dict(name="clip_resnet18_p16", op="clip", P=16, net="resnet18", width=64, depth=1, dtype="fp32", share=0.5),
        # a stack of feed-forward blocks trained in bf16, whose gradients become the fp32 ones of the step
        dict(name="clip_blocks_bf16_p8", op="clip", P=8, net="blocks", width=1024, depth=6, dtype="bf16", share=0.75),
        # one token on each of 4 replicas between two blocks: answering with the trained models
        dict(name="norm_token_bf16", op="residual_norm", P=4, n=1, d=1024, dtype="bf16", train=False),
        # a training step's norm between two blocks, ordinary size
        dict(name="norm_train_bf16", op="residual_norm", P=8, n=1024, d=1024, dtype="bf16", train=True),
        # full precision, ragged token count and a width that is no multiple of a vector
        dict(name="norm_train_fp32_ragged", op="residual_norm", P=3, n=1777, d=1001, dtype="fp32", train=True),
        # the widest rows over the most tokens
        dict(name="norm_train_bf16_wide", op="residual_norm", P=4, n=8192, d=4096, dtype="bf16", train=True),
        # one token on each of 4 replicas: the weights are read for a single row
        dict(name="ffn_token_bf16", op="feed_forward", P=4, n=1, d=1024, f=2816, dtype="bf16", act="silu", train=False),
        # a short ragged prompt in fp16 through the trained block
        dict(name="ffn_prompt_fp16", op="feed_forward", P=2, n=77, d=1024, f=4096, dtype="fp16", act="gelu", train=False),
        # a training step of 8 replicas, ordinary size
        dict(name="ffn_train_bf16", op="feed_forward", P=8, n=512, d=1024, f=2816, dtype="bf16", act="silu", train=True),
        # full precision (the step's own type) at odd sizes
        dict(name="ffn_train_fp32_ragged", op="feed_forward", P=3, n=333, d=509, f=1361, dtype="fp32", act="gelu", train=True),
        # the largest training step
        dict(name="ffn_train_bf16_large", op="feed_forward", P=4, n=4096, d=2048, f=5504, dtype="bf16", act="silu", train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 64 or 8, sometimes odd."""
    w, kind = _log_int(rng, lo, hi), rng.random()
    if kind < 0.45:
        w = max(64, w // 64 * 64)
    else:
        w = w // 8 * 8 if kind < 0.8 else w | 1
    return w if w != 3072 else w + 64


def draw(rng):
    op = rng.choice(["clip", "residual_norm", "feed_forward"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "clip":
        net = rng.choice(["mlp", "resnet18", "blocks"])
        P = _log_int(rng, 1, 16)
        if net == "blocks":
            width = _width(rng, 64, 1024)
            return dict(op=op, P=min(P, 8), net=net, width=width, depth=rng.randint(1, 6), dtype=dtype, share=rng.choice([0.0, 0.5, 1.0]))
        return dict(op=op, P=P, net=net, width=rng.randint(16, 64), depth=1, dtype=dtype, share=rng.choice([0.0, 0.5, 1.0]))
    train = rng.random() < 0.65
    if op == "residual_norm":
        while True:
            P, n, d = _log_int(rng, 1, 16), _log_int(rng, 1, 16384), _width(rng, 64, 8192)
            if P * n * d <= (4 * 8192 * 4096 if dtype != "fp32" else 2 * 8192 * 4096):
                return dict(op=op, P=P, n=n, d=d, dtype=dtype, train=train)
    while True:
        P, n, d = _log_int(rng, 1, 16), _log_int(rng, 1, 8192), _width(rng, 64, 4096)
        f = _width(rng, 2 * d, 4 * d)
        cost = P * n * d * f * (3 if train else 1)
        # relu's derivative is a step: in 32 bits two sums that differ in the last place fall on its two sides
        act = rng.choice(["silu", "gelu", "relu" if dtype != "fp32" else "silu"])
        if cost <= 3 * 4 * 4096 * 2048 * 5504 and 3 * P * d * f <= 3 * 16 * 2048 * 5504:
            return dict(op=op, P=P, n=n, d=d, f=f, dtype=dtype, act=act, train=train)


def _tensor_sizes(net, width, depth):
    """Elements of every tensor of a net, in order."""
    if net == "mlp":
        dims = [784, width, max(1, width // 2), 10]
        return [n for a, b in zip(dims, dims[1:]) for n in (a * b, b)]
    if net == "blocks":  # residual blocks: four vectors of the norms, then gate, up and down
        hidden = width * 11 // 4
        return [n for _ in range(depth) for n in (width, width, width, width, hidden * width, hidden * width, width * hidden)]
    conv = lambda o, i, k: [o * i * k * k, o, o]  # noqa: E731  (a convolution, then scale and shift)
    sizes, inside = conv(width, 3, 3), width
    for stage in range(4):
        w = width << stage
        for b in range(2):
            sizes += conv(w, inside, 3) + conv(w, w, 3)
            if b == 0 and inside != w:
                sizes += conv(w, inside, 1)
            inside = w
    return sizes + [10 * inside, 10]


def _layout(sizes):
    """(offsets, stride): every tensor starts on a 128-byte boundary of fp32 values."""
    offsets, at = [], 0
    for n in sizes:
        offsets.append(at)
        at += -(-n // 32) * 32
    return offsets, at


# ------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, scale, dtype):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _inputs(case, seed):
    """The inputs of a case, from its seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = TYPES[case["dtype"]]
    P = case["P"]
    if case["op"] == "clip":
        sizes = _tensor_sizes(case["net"], case["width"], case["depth"])
        offsets, stride = _layout(sizes)
        g = torch.zeros((P, stride), dtype=dt, device="cuda")
        # replicas meet gradients of different size; `share` of them have a norm over max_norm
        over = [((i * 7 + 3) % P) < case["share"] * P for i in range(P)]
        total = sum(sizes)
        for i in range(P):
            g[i] = _normal(gen, (stride,), (2.5 if over[i] else 0.4) / math.sqrt(total), dt)
        for o, n, after in zip(offsets, sizes, offsets[1:] + [stride]):
            g[:, o + n:after] = 0
        return dict(sizes=sizes, offsets=offsets, grads=g, max_norm=1.0)
    n, d = case["n"], case["d"]
    if case["op"] == "residual_norm":
        s = dict(y=_normal(gen, (P, n, d), 0.7, dt), r=_normal(gen, (P, n, d), 1.3, dt))
        offsets, stride = _layout([d] * 4)
        params = torch.zeros((P, stride), dtype=dt, device="cuda")
        for o, (mean, dev) in zip(offsets, ((1.0, 0.1), (0.0, 1.0), (1.0, 0.1), (1.0, 0.1))):
            params[:, o:o + d] = (mean + _normal(gen, (P, d), dev, torch.float32)).to(dt)
        s.update(offsets=offsets, params=params)
        if case["train"]:
            s.update(d_r=_normal(gen, (P, n, d), 0.1, dt), d_o=_normal(gen, (P, n, d), 0.1, dt))
        return s
    f = case["f"]
    s = dict(x=_normal(gen, (P, n, d), 1.0, dt))
    offsets, stride = _layout([f * d, f * d, d * f])
    params = torch.zeros((P, stride), dtype=dt, device="cuda")
    for o, dev in zip(offsets, (d ** -0.5, d ** -0.5, f ** -0.5)):
        for i in range(P):
            params[i, o:o + f * d] = _normal(gen, (f * d,), dev, dt)
    s.update(offsets=offsets, params=params)
    if case["train"]:
        s.update(dy=_normal(gen, (P, n, d), 0.2, dt))
    return s


def _views(case, buffer, offsets):
    """The tensors of a ``[P, stride]`` buffer as a caller holds them."""
    P, d = case["P"], case["d"]
    if case["op"] == "residual_norm":
        return [buffer[:, o:o + d] for o in offsets]
    f = case["f"]
    return [buffer[:, o:o + f * d].view(P, *shape) for o, shape in zip(offsets, ((f, d), (f, d), (d, f)))]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":
        s["out"] = torch.zeros(s["grads"].shape, dtype=torch.float32, device="cuda")
        if own:
            from paper_2103_07454_b200 import binding
            s["ring"] = binding.EventGrad(case["P"], s["sizes"])
            assert s["ring"].tensor_offset == s["offsets"]
    else:
        s["weights"] = _views(case, s["params"], s["offsets"])
        if case["train"]:  # the buffer of gradients that the step reads
            s["grads"] = torch.zeros_like(s["params"])
            s["d_weights"] = _views(case, s["grads"], s["offsets"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"clip": _own_clip, "residual_norm": _own_norm, "feed_forward": _own_ffn}[op](s)
    return {"clip": _plain_clip, "residual_norm": _plain_norm, "feed_forward": _plain_ffn}[op](s)


def _own_clip(s):
    norms = s["ring"].clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    return dict(norms=norms, grads=s["out"])


def _own_norm(s):
    from paper_2103_07454_b200 import binding
    w_post, gate, scale, w_pre = s["weights"]
    r_out, o = binding.residual_norm(s["y"], s["r"], w_post=w_post, gate=gate, scale=scale, w_pre=w_pre, eps=EPS)
    if not s["case"]["train"]:
        return dict(r=r_out, o=o)
    dy, dr, _ = binding.residual_norm_backward(s["d_r"], s["d_o"], s["y"], s["r"], w_post=w_post, gate=gate, scale=scale,
                                               w_pre=w_pre, eps=EPS, d_weights=s["d_weights"])
    return dict(r=r_out, o=o, dy=dy, dr=dr, dw=s["grads"])


def _own_ffn(s):
    from paper_2103_07454_b200 import binding
    act = s["case"]["act"]
    if not s["case"]["train"]:
        return dict(y=binding.feed_forward(s["x"], *s["weights"], activation=act))
    y, saved = binding.feed_forward(s["x"], *s["weights"], activation=act, save=True)
    dx, _ = binding.feed_forward_backward(s["dy"], s["x"], *s["weights"], saved, activation=act, d_weights=s["d_weights"])
    return dict(y=y, dx=dx, dw=s["grads"])


def _plain_clip(s):
    g = s["grads"].float()
    norms = (g * g).sum(1).sqrt()
    torch.mul(g, (s["max_norm"] / norms).clamp(max=1.0)[:, None], out=s["out"])
    return dict(norms=norms, grads=s["out"])


def _plain_norm(s):
    dt = s["y"].dtype
    y, r = s["y"].float(), s["r"].float()
    w_post, gate, scale, w_pre = (w.float()[:, None, :] for w in s["weights"])
    inv1 = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    yh = y * inv1
    u = yh * w_post
    sg = 1.0 / (1.0 + torch.exp(-gate))
    rn = scale * r + sg * u
    inv2 = torch.rsqrt((rn * rn).mean(-1, keepdim=True) + EPS)
    rh = rn * inv2
    out = dict(r=rn.to(dt), o=(rh * w_pre).to(dt))
    if not s["case"]["train"]:
        return out
    d_r, d_o = s["d_r"].float(), s["d_o"].float()
    dn = d_o * w_pre
    dR = d_r + inv2 * (dn - rh * (dn * rh).mean(-1, keepdim=True))
    du = sg * dR
    dyh = du * w_post
    dy = inv1 * (dyh - yh * (dyh * yh).mean(-1, keepdim=True))
    sums = ((du * yh).sum(1), (dR * u * sg * (1.0 - sg)).sum(1), (dR * r).sum(1), (d_o * rh).sum(1))
    for to, v in zip(s["d_weights"], sums):
        to.copy_(v)
    return dict(out, dy=dy.to(dt), dr=(scale * dR).to(dt), dw=s["grads"])


def _plain_act(name, g):
    """act(g) and its derivative."""
    if name == "relu":
        on = (g > 0).float()
        return g * on, on
    if name == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_ffn(s):
    dt = s["x"].dtype
    x = s["x"].float()
    wg, wu, wd = (w.float() for w in s["weights"])
    g, u = x @ wg.transpose(1, 2), x @ wu.transpose(1, 2)
    a, da = _plain_act(s["case"]["act"], g)
    h = a * u
    y = (h @ wd.transpose(1, 2)).to(dt)
    if not s["case"]["train"]:
        return dict(y=y)
    dy = s["dy"].float()
    dh = dy @ wd
    du, dg = dh * a, dh * u * da
    dx = (dg @ wg + du @ wu).to(dt)
    sums = (dg.transpose(1, 2) @ x, du.transpose(1, 2) @ x, dy.transpose(1, 2) @ h)
    for to, v in zip(s["d_weights"], sums):
        to.copy_(v)
    return dict(y=y, dx=dx, dw=s["grads"])


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What ``run`` returns, in 64 bits from the definitions; the gradients by differentiating the forward pass."""
    s = _inputs(case, seed)
    if case["op"] == "clip":
        g, out, norms = s["grads"], torch.zeros(s["grads"].shape, dtype=torch.float64, device="cuda"), []
        for i in range(case["P"]):
            sq = sum(float(g[i, o:o + n].double().pow(2).sum()) for o, n in zip(s["offsets"], s["sizes"]))
            norms.append(math.sqrt(sq))
            out[i] = g[i].double() * (s["max_norm"] / norms[-1] if norms[-1] > s["max_norm"] else 1.0)
        return dict(norms=torch.tensor(norms, dtype=torch.float64), grads=out)
    train = case["train"]
    params = s["params"].double().requires_grad_(train)
    dw = torch.zeros_like(s["params"], dtype=torch.float64)
    names, grads_of = ("r", "o"), ("y", "r")
    if case["op"] == "feed_forward":
        names, grads_of = ("y",), ("x",)
    outs, d_ins = {k: [] for k in names}, {k: [] for k in grads_of}
    for i in range(case["P"]):  # one replica at a time, to keep the memory small
        one = dict(case, P=1)
        ins = {k: s[k][i:i + 1].double().requires_grad_(train) for k in grads_of}
        row = params[i:i + 1].detach().requires_grad_(train)
        w = _views(one, row, s["offsets"])
        if case["op"] == "residual_norm":
            rms = lambda v: v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / v.shape[-1] + EPS)  # noqa: E731
            res = w[2].unsqueeze(1) * ins["r"] + torch.sigmoid(w[1]).unsqueeze(1) * (rms(ins["y"]) * w[0].unsqueeze(1))
            result = (res, rms(res) * w[3].unsqueeze(1))
            given = (s["d_r"], s["d_o"]) if train else ()
        else:
            g = torch.einsum("pnd,pfd->pnf", ins["x"], w[0])
            a = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[case["act"]](g)
            result = (torch.einsum("pnf,pdf->pnd", a * torch.einsum("pnd,pfd->pnf", ins["x"], w[1]), w[2]),)
            given = (s["dy"],) if train else ()
        for k, v in zip(names, result):
            outs[k].append(v.detach())
        if train:
            got = torch.autograd.grad(result, [ins[k] for k in grads_of] + [row], [v[i:i + 1].double() for v in given])
            for k, v in zip(grads_of, got):
                d_ins[k].append(v)
            dw[i:i + 1] = got[-1]
    out = {k: torch.cat(v) for k, v in outs.items()}
    if train:
        out.update({"d" + k: torch.cat(v) for k, v in d_ins.items()}, dw=dw)
    return out


# ------------------------------------------------------------------------------------------ the least work
def work(case):
    P, b = case["P"], torch.finfo(TYPES[case["dtype"]]).bits // 8
    if case["op"] == "clip":
        n = P * sum(_tensor_sizes(case["net"], case["width"], case["depth"]))
        return {"bytes": n * (b + 4), "flops": 3 * n}
    n, d = case["n"], case["d"]
    if case["op"] == "residual_norm":
        # forward: y, r in and r', o out; a training pass also reads d_r', d_o and writes dy, dr
        rows, vectors = (8, 8) if case["train"] else (4, 4)
        return {"bytes": P * b * d * (rows * n + vectors), "flops": P * n * d * (45 if case["train"] else 12)}
    f = case["f"]
    if case["train"]:  # x, dy in, y, dx out; three weights in and their gradients out
        return {"bytes": P * b * (4 * n * d + 6 * d * f), "flops": 18 * P * n * d * f}
    return {"bytes": P * b * (2 * n * d + 3 * d * f), "flops": 6 * P * n * d * f}
