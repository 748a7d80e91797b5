"""What a ring of replicas needs around its blocks to train a language model, as cases that can be timed and checked.

P replicas, each with weights of its own, read tokens, rotate the queries and keys of their attention heads by position, and
turn the gradients of their matrices into orthogonal updates before the event-triggered step takes them:

* ``embedding``      y[i] = scale * W[token i], and its gradient dW[v] = scale * sum of dy over the places of token v;
* ``head_norm``      rms norm of every head of the queries and keys, then the rotation by position, and the gradients;
* ``orthogonalise``  X = u / |u|, a few times X = a X + (b X X^T + c (X X^T)^2) X, of every matrix of every replica, u being
                     the gradient or what momentum makes of it.

Weights and gradients are views into ``[P, stride]`` buffers, tensor after tensor, each on a 128-byte boundary of fp32
parameters: the layout that the step works on.  ``own`` False computes the operators in their plain form.
"""
import math

import torch

own = False

EPS = 1e-6
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token on each of 4 replicas, answering with the trained models: a call bound by its latency
        dict(name="embedding_token_bf16", op="embedding", P=4, n=1, V=32000, d=1024, dtype="bf16", pad=0.0, train=False),
        # full precision, odd width, sequences padded with tokens that are none
        dict(name="embedding_train_fp32_ragged", op="embedding", P=3, n=777, V=1009, d=509, dtype="fp32", pad=0.2, train=True),
        # a training step of ordinary size: most rows of the table take no gradient
        dict(name="embedding_train_bf16", op="embedding", P=8, n=1024, V=32000, d=1024, dtype="bf16", pad=0.0, train=True),
        # the most tokens over the widest rows: the frequent ones come thousands of times
        dict(name="embedding_train_bf16_large", op="embedding", P=4, n=16384, V=32000, d=2048, dtype="bf16", pad=0.05, train=True),
        # one token on each of 4 replicas, far into its sequence
        dict(name="head_norm_token_bf16", op="head_norm", P=4, n=1, hq=16, hk=4, dh=64, rotary=64, interleaved=False, far=100000,
             dtype="bf16", train=False),
        # a training step of ordinary size, queries and keys as parts of one projection
        dict(name="head_norm_train_bf16", op="head_norm", P=8, n=1024, hq=16, hk=4, dh=64, rotary=64, interleaved=False, far=0,
             dtype="bf16", train=True),
        # full precision, ragged token count, neighbours rotated, a part of every head left as it is
        dict(name="head_norm_train_fp32_ragged", op="head_norm", P=3, n=777, hq=5, hk=5, dh=90, rotary=46, interleaved=True, far=5000,
             dtype="fp32", train=True),
        # the largest training step
        dict(name="head_norm_train_bf16_large", op="head_norm", P=4, n=8192, hq=16, hk=4, dh=128, rotary=128, interleaved=False,
             far=0, dtype="bf16", train=True),
        # the matrices of the small 784-64-32-10 perceptron on 4 replicas: many short products, one after another
        dict(name="orthogonalise_mlp_p4", op="orthogonalise", P=4, net="mlp", rows=64, cols=0, depth=1, dtype="fp32", steps=5,
             momentum=0.95, nesterov=True),
        # the convolutions of a ResNet-18 as matrices, on 8 replicas in the step's own type
        dict(name="orthogonalise_resnet18_p8", op="orthogonalise", P=8, net="resnet18", rows=64, cols=0, depth=1, dtype="fp32",
             steps=5, momentum=0.95, nesterov=True),
        # two feed-forward blocks of ordinary size on 8 replicas, trained in bf16
        dict(name="orthogonalise_blocks_bf16_p8", op="orthogonalise", P=8, net="blocks", rows=1024, cols=2816, depth=2, dtype="bf16",
             steps=5, momentum=0.0, nesterov=False),
        # the largest: the feed-forward block of the largest training step
        dict(name="orthogonalise_large_bf16", op="orthogonalise", P=4, net="blocks", rows=2048, cols=5504, depth=1, dtype="bf16",
             steps=5, momentum=0.95, nesterov=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: mostly a multiple of 64 or 8, sometimes odd."""
    w, kind = _log_int(rng, lo, hi), rng.random()
    if kind < 0.45:
        return max(64, w // 64 * 64)
    return max(8, w // 8 * 8) if kind < 0.8 else w | 1


def draw(rng):
    op = rng.choice(["embedding", "head_norm", "orthogonalise"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    half = 2 if dtype == "fp32" else 1                      # values of four bytes: half as many
    if op == "embedding":
        while True:
            P, n, V, d = _log_int(rng, 1, 16), _log_int(rng, 1, 16384), _log_int(rng, 64, 65536), _width(rng, 32, 4096)
            if P * n * d * half <= 4 * 16384 * 2048 and P * V * d * half <= 4 * 32000 * 2048:
                return dict(op=op, P=P, n=n, V=V, d=d, dtype=dtype, pad=rng.choice([0.0, 0.1, 0.5]), train=rng.random() < 0.7)
    if op == "head_norm":
        while True:
            P, n, hk = _log_int(rng, 1, 16), _log_int(rng, 1, 16384), rng.choice([1, 2, 3, 4, 8])
            hq, dh = hk * rng.choice([1, 2, 4, 7]), rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256, rng.randint(9, 160)])
            rotary = rng.choice([dh, dh, dh // 2, dh // 4]) // 2 * 2
            if P * n * (hq + 2 * hk) * dh * half <= 4 * 8192 * 24 * 128:
                return dict(op=op, P=P, n=n, hq=hq, hk=hk, dh=dh, rotary=rotary, interleaved=rng.random() < 0.3,
                            far=rng.choice([0, 0, 3000, 1000000]), dtype=dtype, train=rng.random() < 0.7)
    while True:
        net = rng.choice(["mlp", "resnet18", "blocks", "single"])
        c = dict(op=op, P=_log_int(rng, 1, 16), net=net, rows=0, cols=0, depth=1, dtype=dtype, steps=rng.choice([3, 5, 5, 6]),
                 momentum=rng.choice([0.0, 0.9, 0.95]), nesterov=rng.random() < 0.5)
        if net in ("mlp", "resnet18"):
            c["rows"] = rng.randint(16, 64)
        elif net == "blocks":
            c.update(rows=_width(rng, 64, 2048), depth=rng.randint(1, 3))
            c["cols"] = _width(rng, 2 * c["rows"], 4 * c["rows"])
        else:
            c.update(rows=_width(rng, 8, 4096), cols=_width(rng, 8, 4096))
        cost = sum(min(a, b) ** 2 * max(a, b) for a, b in _matrices(c)) * c["P"] * c["steps"] / 5
        elements = sum(a * b for a, b in _matrices(c)) * c["P"]
        # products of full precision take three times as long on the tensor cores
        if cost * (3 if dtype != "bf16" else 1) <= 12 * 2048 ** 2 * 5504 and elements * half <= 12 * 2048 * 5504:
            return c


def _matrices(case):
    """(rows, columns) of the matrices of a net."""
    net, w = case["net"], case["rows"]
    if net == "mlp":
        dims = [784, w, max(1, w // 2), 10]
        return [(b, a) for a, b in zip(dims, dims[1:])]
    if net == "blocks":
        return [(case["cols"], w), (case["cols"], w), (w, case["cols"])] * case["depth"]
    if net == "single":
        return [(w, case["cols"])]
    shapes, inside = [(w, 27)], w
    for stage in range(4):
        out = w << stage
        for b in range(2):
            shapes += [(out, inside * 9), (out, out * 9)]
            if b == 0 and inside != out:
                shapes.append((out, inside))
            inside = out
    return shapes + [(10, inside)]


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
    dt, P = TYPES[case["dtype"]], case["P"]
    if case["op"] == "orthogonalise":
        return _gradients(case, gen, dt)
    n = case["n"]
    if case["op"] == "embedding":
        V, d = case["V"], case["d"]
        # how often a token comes falls with its number, as words do; the end of a sequence holds no tokens
        u = torch.rand((P, n), generator=gen, device="cuda", dtype=torch.float64)
        tokens = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
        if case["pad"] > 0:
            lengths = n - (torch.rand((P, 1), generator=gen, device="cuda") * 2 * case["pad"] * n).long()
            tokens[torch.arange(n, device="cuda")[None, :] >= lengths] = -1
        offsets, stride = _layout([V * d])
        params = torch.zeros((P, stride), dtype=dt, device="cuda")
        for i in range(P):
            params[i, :V * d] = _normal(gen, (V * d,), 0.02, dt)
        s = dict(tokens=tokens, params=params, offsets=offsets)
        if case["train"]:
            s["dy"] = _normal(gen, (P, n, d), 0.1, dt)
        return s
    hq, hk, dh = case["hq"], case["hk"], case["dh"]
    heads = hq + 2 * hk
    if n == 1:
        positions = torch.randint(0, case["far"] + 1, (P, 1), generator=gen, device="cuda")
    else:  # two documents in a row, the second one's places counted from `far`
        cut = torch.randint(1, n, (P, 1), generator=gen, device="cuda")
        at = torch.arange(n, device="cuda")[None, :].expand(P, n)
        positions = torch.where(at < cut, at, at - cut + case["far"])
    s = dict(positions=positions.contiguous(), qkv=_normal(gen, (P, n, heads * dh), 1.3, dt))
    offsets, stride = _layout([dh, dh])
    params = torch.zeros((P, stride), dtype=dt, device="cuda")
    for o in offsets:
        params[:, o:o + dh] = (1.0 + _normal(gen, (P, dh), 0.1, torch.float32)).to(dt)
    s.update(params=params, offsets=offsets)
    if case["train"]:
        s.update(dq_out=_normal(gen, (P, n, hq, dh), 0.1, dt), dk_out=_normal(gen, (P, n, hk, dh), 0.1, dt))
    return s


def _gradients(case, gen, dt):
    """Gradients of matrices: a few directions of falling weight, as a batch leaves them, over noise."""
    P, shapes = case["P"], _matrices(case)
    offsets, stride = _layout([a * b for a, b in shapes])
    grads = torch.zeros((P, stride), dtype=dt, device="cuda")
    velocity = torch.zeros((P, stride), dtype=torch.float32, device="cuda") if case["momentum"] else None
    for o, (a, b) in zip(offsets, shapes):
        k = min(a, b, 16)
        weights = torch.logspace(0.5, -1.0, k, device="cuda") / math.sqrt(k)
        for to in (grads, velocity):
            if to is None:
                continue
            for i in range(P):
                left, right = _normal(gen, (a, k), 1.0, torch.float32), _normal(gen, (k, b), 1.0, torch.float32)
                value = (left * weights) @ right + _normal(gen, (a, b), 0.5, torch.float32)
                to[i, o:o + a * b] = (value * 1e-3).to(to.dtype).reshape(-1)
    return dict(shapes=shapes, offsets=offsets, grads=grads, velocity=velocity)


def _views(s, buffer, shapes):
    """The tensors of a ``[P, stride]`` buffer as a caller holds them."""
    return [buffer[:, o:o + math.prod(shape)].view(buffer.shape[0], *shape) for o, shape in zip(s["offsets"], shapes)]


def _heads(case, buffer):
    """Queries and keys of a projection ``[P, n, (hq + 2 hk) * dh]``."""
    P, n, hq, hk, dh = (case[k] for k in ("P", "n", "hq", "hk", "dh"))
    heads = buffer.view(P, n, hq + 2 * hk, dh)
    return heads[:, :, :hq], heads[:, :, hq:hq + hk]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "orthogonalise":
        s["out"] = torch.zeros_like(s["grads"])
        s["d_views"], s["out_views"] = _views(s, s["grads"], s["shapes"]), _views(s, s["out"], s["shapes"])
        if s["velocity"] is not None:
            s["velocity_out"] = torch.zeros_like(s["velocity"])
            s["v_views"], s["vo_views"] = (_views(s, s[k], s["shapes"]) for k in ("velocity", "velocity_out"))
        return s
    shapes = [(case["V"], case["d"])] if case["op"] == "embedding" else [(case["dh"],)] * 2
    s["weights"] = _views(s, s["params"], shapes)
    if case["op"] == "head_norm":
        s["q"], s["k"] = _heads(case, s["qkv"])
    if case["train"]:  # the buffer of gradients that the step reads
        s["grads"] = torch.zeros_like(s["params"])
        s["d_weights"] = _views(s, s["grads"], shapes)
        if case["op"] == "head_norm":  # the projection's gradient, whose last part attention fills
            s["d_qkv"] = torch.zeros_like(s["qkv"])
            s["dq"], s["dk"] = _heads(case, s["d_qkv"])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"embedding": _own_embedding, "head_norm": _own_heads, "orthogonalise": _own_orthogonalise}[op](s)
    return {"embedding": _plain_embedding, "head_norm": _plain_heads, "orthogonalise": _plain_orthogonalise}[op](s)


def _own_embedding(s):
    from paper_2103_07454_b200 import binding
    scale = math.sqrt(s["case"]["d"])
    y = binding.embedding(s["tokens"], s["weights"][0], scale=scale)
    if not s["case"]["train"]:
        return dict(y=y)
    binding.embedding_backward(s["dy"], s["tokens"], scale=scale, d_weight=s["d_weights"][0])
    return dict(y=y, dw=s["grads"])


def _own_heads(s):
    from paper_2103_07454_b200 import binding
    c = s["case"]
    w_q, w_k = s["weights"]
    how = dict(w_q=w_q, w_k=w_k, positions=s["positions"], rotary=c["rotary"], interleaved=c["interleaved"], eps=EPS)
    q, k = binding.head_norm(s["q"], s["k"], **how)
    if not c["train"]:
        return dict(q=q, k=k)
    binding.head_norm_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], dq=s["dq"], dk=s["dk"], d_weights=s["d_weights"], **how)
    return dict(q=q, k=k, d_qkv=s["d_qkv"], dw=s["grads"])


def _own_orthogonalise(s):
    from paper_2103_07454_b200 import binding
    c = s["case"]
    if s["velocity"] is None:
        binding.orthogonalise(s["d_views"], out=s["out_views"], steps=c["steps"])
        return dict(out=s["out"])
    binding.orthogonalise(s["d_views"], out=s["out_views"], steps=c["steps"], velocity=s["v_views"], velocity_out=s["vo_views"],
                          momentum=c["momentum"], nesterov=c["nesterov"])
    return dict(out=s["out"], velocity=s["velocity_out"])


def _plain_embedding(s):
    c, w, tokens = s["case"], s["weights"][0], s["tokens"]
    P, n, V, d, scale = c["P"], c["n"], c["V"], c["d"], math.sqrt(c["d"])
    there = ((tokens >= 0) & (tokens < V))[:, :, None]
    replica = torch.arange(P, device="cuda")[:, None]
    y = (w[replica, tokens.clamp(0, V - 1)].float() * scale * there).to(w.dtype)
    if not c["train"]:
        return dict(y=y)
    rows = torch.zeros((P * V, d), dtype=torch.float32, device="cuda")
    rows.index_add_(0, (replica * V + tokens.clamp(0, V - 1)).view(-1), (s["dy"].float() * there).view(P * n, d))
    s["d_weights"][0].copy_(rows.view(P, V, d) * scale)
    return dict(y=y, dw=s["grads"])


def _plain_turn(c, positions):
    """Cosine and sine of every place's angles, ``[P, n, 1, rotary / 2]``."""
    pairs = torch.arange(c["rotary"] // 2, device="cuda", dtype=torch.float64)
    angle = positions.double()[:, :, None, None] * 10000.0 ** (-2.0 * pairs / max(1, c["rotary"]))
    return torch.cos(angle).float(), torch.sin(angle).float()


def _plain_rotate(c, x, cos, sin):
    r = c["rotary"]
    out = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., first], x[..., second]
    out[..., first] = a * cos - b * sin
    out[..., second] = a * sin + b * cos
    return out


def _plain_heads(s):
    c = s["case"]
    cos, sin = _plain_turn(c, s["positions"])
    out = {}
    for name, x, w, d_out, dx, dw in zip("qk", (s["q"], s["k"]), s["weights"], (s.get("dq_out"), s.get("dk_out")),
                                         (s.get("dq"), s.get("dk")), s.get("d_weights", (None, None))):
        v, wide = x.float(), w.float()[:, None, None, :]
        inv = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
        vh = v * inv
        out[name] = _plain_rotate(c, vh * wide, cos, sin).to(x.dtype)
        if not c["train"]:
            continue
        dz = _plain_rotate(c, d_out.float(), cos, -sin)
        dvh = dz * wide
        dx.copy_(inv * (dvh - vh * (dvh * vh).mean(-1, keepdim=True)))
        dw.copy_((dz * vh).sum((1, 2)))
    return dict(out, d_qkv=s["d_qkv"], dw=s["grads"]) if c["train"] else out


def _plain_orthogonalise(s):
    c = s["case"]
    a, b, k = COEFFICIENTS
    for j, (g, to) in enumerate(zip(s["d_views"], s["out_views"])):
        u = g.float()
        if s["velocity"] is not None:
            v = c["momentum"] * s["v_views"][j] + u
            s["vo_views"][j].copy_(v)
            u = u + c["momentum"] * v if c["nesterov"] else v
        tall = u.shape[1] > u.shape[2]
        x = u.transpose(1, 2) if tall else u
        x = x / x.pow(2).sum((1, 2), keepdim=True).sqrt()
        for _ in range(c["steps"]):
            gram = x @ x.transpose(1, 2)
            x = a * x + (b * gram + k * (gram @ gram)) @ x
        to.copy_(x.transpose(1, 2) if tall else x)
    return dict(out=s["out"]) if s["velocity"] is None else dict(out=s["out"], velocity=s["velocity_out"])


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What ``run`` returns, in 64 bits from the definitions; the gradients by differentiating the forward pass."""
    s = _inputs(case, seed)
    if case["op"] == "orthogonalise":
        return _exact_orthogonalise(case, s)
    P, n, train = case["P"], case["n"], case["train"]
    dw = torch.zeros_like(s["params"], dtype=torch.float64)
    outs = {}
    if case["op"] == "embedding":
        V, d = case["V"], case["d"]
        y = torch.zeros((P, n, d), dtype=torch.float64, device="cuda")
        for i in range(P):
            row = s["params"][i:i + 1].double().requires_grad_(train)
            at = torch.nonzero(s["tokens"][i] >= 0)[:, 0]
            got = _views(s, row, [(V, d)])[0][0].index_select(0, s["tokens"][i, at]).mul(math.sqrt(d))
            y[i].index_copy_(0, at, got.detach())
            if train:
                dw[i:i + 1] = torch.autograd.grad(got, row, s["dy"][i, at].double())[0]
        return dict(y=y, dw=dw) if train else dict(y=y)
    r, dh = case["rotary"], case["dh"]
    names = {"q": "dq_out", "k": "dk_out"}
    d_qkv = torch.zeros_like(s["qkv"], dtype=torch.float64)
    for i in range(P):
        row = s["params"][i:i + 1].double().requires_grad_(train)
        qkv = s["qkv"][i:i + 1].double().requires_grad_(train)
        exponents = torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / max(1, r)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           s["positions"][i].double()[:, None, None] / torch.pow(10000.0, exponents))
        results = []
        for v, w in zip(_heads(dict(case, P=1), qkv), _views(s, row, [(dh,)] * 2)):
            v = v[0]
            z = v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / dh + EPS) * w[0]
            lead, rest = z[..., :r], z[..., r:]
            pairs = lead.unflatten(-1, (r // 2, 2)) if case["interleaved"] else lead.unflatten(-1, (2, r // 2)).transpose(-1, -2)
            turned = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
            results.append(torch.cat([(turned if case["interleaved"] else turned.transpose(-1, -2)).flatten(-2), rest], -1))
        for name, v in zip(names, results):
            outs.setdefault(name, []).append(v.detach())
        if train:
            given = [s[names[name]][i].double() for name in names]
            d_qkv[i:i + 1], dw[i:i + 1] = torch.autograd.grad(results, [qkv, row], given)
    outs = {name: torch.stack(v) for name, v in outs.items()}
    return dict(outs, d_qkv=d_qkv, dw=dw) if train else outs


def _exact_orthogonalise(case, s):
    a, b, c = COEFFICIENTS
    out = torch.zeros_like(s["grads"], dtype=torch.float64)
    u, velocity = s["grads"].double(), None
    if s["velocity"] is not None:
        velocity = s["velocity"].double().mul(case["momentum"]).add(u)
        u = torch.add(u, velocity, alpha=case["momentum"]) if case["nesterov"] else velocity
    for given, to in zip(_views(s, u, s["shapes"]), _views(s, out, s["shapes"])):
        for x, y in zip(given, to):
            flip = x.shape[0] > x.shape[1]
            x = (x.T if flip else x) / torch.linalg.matrix_norm(x)
            eye = torch.eye(x.shape[0], dtype=torch.float64, device="cuda")
            for _ in range(case["steps"]):
                gram = torch.mm(x, x.T)
                x = torch.mm(a * eye + torch.mm(b * eye + c * gram, gram), x)
            y.copy_(x.T if flip else x)
    return dict(out=out) if velocity is None else dict(out=out, velocity=velocity)


# ------------------------------------------------------------------------------------------ the least work
def work(case):
    P, b = case["P"], torch.finfo(TYPES[case["dtype"]]).bits // 8
    if case["op"] == "orthogonalise":
        elements = sum(r * c for r, c in _matrices(case))
        # two of the three products of a step are symmetric: half of their elements are enough
        flops = sum(3 * min(m) ** 2 * max(m) + min(m) ** 3 for m in _matrices(case)) * case["steps"]
        return {"bytes": P * elements * (2 * b + (8 if case["momentum"] else 0)), "flops": P * flops}
    n = case["n"]
    if case["op"] == "embedding":
        V, d = case["V"], case["d"]
        # distinct tokens of a sequence: their rows in, and all of dy; y out and the whole table's gradient
        kinds = min(V, n)
        nbytes = P * (8 * n + b * d * (kinds + n))
        if case["train"]:
            nbytes += P * (8 * n + b * d * (n + V))
        return {"bytes": nbytes, "flops": P * n * d * (3 if case["train"] else 1)}
    values = P * n * (case["hq"] + case["hk"]) * case["dh"]
    # forward: heads in and out; a training pass also reads them again with their gradients and writes the gradients
    return {"bytes": values * b * (5 if case["train"] else 2), "flops": values * (30 if case["train"] else 10)}
