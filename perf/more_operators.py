"""What is measured of the two ends of a training step: the loss over a large vocabulary with its gradient, and the update
whose singular values are brought near one.

`run` computes each operator in its plain form (elementary torch operations in 32 bits) or, with `own` set, by this
package's calls; `exact` computes it in 64 bits.

  loss            z = h w^T (h [tokens][width], w [vocabulary][width]); loss_t = log sum_v exp z_tv - z_t,y; 0 where y = IGNORED
  train           the loss and, for a gradient g_t of each loss, dh = dz w and dw = dz^T h, dz_tv = g_t (softmax(z_t)_v - [v = y])
  orthogonalise   X = U / |U|_F, then five times X <- a X + (b A + c A^2) X with A = X X^T (or the same from the right,
                  X (b A + c A^2) with A = X^T X, which is equal)
  step            m <- beta m + (1 - beta) g;  u = m, or beta m + (1 - beta) g;  x <- x - delta orthogonalise(u)
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
IGNORED = -100
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
BETA, DELTA = 0.95, 0.02


def listed():
    return [
        # a handful of tokens of a toy model: a call of a few microseconds
        {"name": "loss 8x1000x64 f16", "op": "loss", "tokens": 8, "vocab": 1000, "width": 64, "type": "f16", "ignored": 0.0},
        # one token scored over the BERT-large-sized vocabulary: the weight's bytes
        {"name": "loss 1x30522x1024 bf16", "op": "loss", "tokens": 1, "vocab": 30522, "width": 1024, "type": "bf16", "ignored": 0.0},
        # evaluation over a vocabulary whose logits would be 1 GB in 16 bits
        {"name": "loss 4096x131072x2048 f16", "op": "loss", "tokens": 4096, "vocab": 131072, "width": 2048, "type": "f16", "ignored": 0.1},
        # a mini-batch of sides that no tile divides, rows that start off 16 bytes
        {"name": "train 777x5003x1111 f16", "op": "train", "tokens": 777, "vocab": 5003, "width": 1111, "type": "f16", "ignored": 0.3},
        # the BERT-large-sized head in training, a tenth of the batch padding
        {"name": "train 2048x30522x1024 bf16", "op": "train", "tokens": 2048, "vocab": 30522, "width": 1024, "type": "bf16", "ignored": 0.1},
        # a large head in training, where the tensor cores are the bound
        {"name": "train 8192x32768x4096 bf16", "op": "train", "tokens": 8192, "vocab": 32768, "width": 4096, "type": "bf16", "ignored": 0.05},
        # a layer of the toy perceptron: latency
        {"name": "orthogonalise 64x64 f32", "op": "orthogonalise", "count": 1, "rows": 64, "cols": 64, "type": "f32", "out": "f32"},
        # the feed-forward matrices of the BERT-large-sized model, one call for the 24 blocks
        {"name": "orthogonalise 24x1024x4096", "op": "orthogonalise", "count": 24, "rows": 1024, "cols": 4096, "type": "bf16", "out": "bf16"},
        # one large square matrix
        {"name": "orthogonalise 4096x4096", "op": "orthogonalise", "count": 1, "rows": 4096, "cols": 4096, "type": "bf16", "out": "bf16"},
        # a tall matrix of odd sides, bf16 gradients, looking ahead
        {"name": "step 1999x503 bf16 ahead", "op": "step", "count": 1, "rows": 1999, "cols": 503, "type": "bf16", "ahead": True},
        # the attention matrices of the BERT-large-sized model, one call for the 24 blocks
        {"name": "step 24x1024x1024 f32", "op": "step", "count": 24, "rows": 1024, "cols": 1024, "type": "f32", "ahead": False},
        # a large layer taller than wide
        {"name": "step 8192x2048 f32", "op": "step", "count": 1, "rows": 8192, "cols": 2048, "type": "f32", "ahead": False},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n // 32 * 32 if rng.random() < 0.5 and n > 64 else n

    op = rng.choice(["loss", "train", "orthogonalise", "step"])
    if op in ("loss", "train"):
        c = {"op": op, "tokens": size(1, 8192), "vocab": size(100, 131072), "width": size(32, 6000), "type": rng.choice(["bf16", "f16"]),
             "ignored": rng.choice([0.0, 0.1, 0.5])}
        while c["tokens"] * c["vocab"] > 300_000_000 or c["tokens"] * c["vocab"] * c["width"] > 600_000_000_000:
            c["tokens"] = c["tokens"] * 2 // 3
        return c
    c = {"op": op, "count": rng.choice([1, 1, size(1, 30)]), "rows": size(16, 8192), "cols": size(16, 8192), "type": rng.choice(["f32", "bf16", "f16"])}
    while c["count"] > 1 and work({**c, "out": "f32"})["flops"] > 1.2e12:
        c["count"] = c["count"] // 2
    while work({**c, "out": "f32"})["flops"] > 1.2e12:
        c["rows"], c["cols"] = c["rows"] * 2 // 3, c["cols"] * 2 // 3
    if op == "step":
        return {**c, "ahead": rng.random() < 0.5}
    return {**c, "out": rng.choice(["bf16", "f32"])}


def work(case):
    if case["op"] in ("loss", "train"):
        t, v, d, e = case["tokens"], case["vocab"], case["width"], BYTES[case["type"]]
        ways = 1 if case["op"] == "loss" else 2           # h and w in, dh and dw out
        return {"bytes": ways * e * d * (t + v) + 12 * t, "flops": (2 if case["op"] == "loss" else 6) * t * v * d}
    n, r, c = case["count"], case["rows"], case["cols"]
    s = min(r, c)
    e = BYTES[case["type"]] + (BYTES[case["out"]] if case["op"] == "orthogonalise" else 16)      # x and m are read and written
    # A and A^2 are symmetric: half of each
    return {"bytes": n * r * c * e, "flops": n * STEPS * (r * c * s + s ** 3 + 2 * r * c * s)}


# --------------------------------------------------------------------------------------------------------------------
# inputs


def _gen(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + key) & (2**62 - 1))
    return g


def _update(n, r, c, gen):
    """Momentum-like matrices: a few strong directions over noise, rows and columns of different sizes."""
    u = torch.randn(n, r, c, generator=gen, device="cuda")
    k = max(1, min(r, c) // 16)
    strong = torch.matmul(torch.randn(n, r, k, generator=gen, device="cuda"), torch.randn(n, k, c, generator=gen, device="cuda"))
    u += strong.mul_(1.5 / k ** 0.5)
    u *= torch.exp(0.5 * torch.randn(n, r, 1, generator=gen, device="cuda"))
    u *= torch.exp(0.5 * torch.randn(n, 1, c, generator=gen, device="cuda"))
    return u.mul_(1e-3)


def prepare(case, seed):
    s = {"case": case}
    if case["op"] in ("loss", "train"):
        t, v, d = case["tokens"], case["vocab"], case["width"]
        gen = _gen(seed, 1)
        w = torch.randn(v, d, generator=gen, device="cuda").mul_(0.02)
        y = torch.randint(0, v, (t,), generator=gen, device="cuda")
        h = torch.randn(t, d, generator=gen, device="cuda")
        # tokens from unsure to sure: up to 12 is added to the target's logit
        lean = 12 * torch.rand(t, 1, generator=gen, device="cuda")
        h += lean * w[y] / w[y].square().sum(1, keepdim=True)
        ignored = torch.rand(t, generator=gen, device="cuda") < case["ignored"]
        s["h"], s["w"] = h.to(TYPES[case["type"]]), w.to(TYPES[case["type"]])
        s["y"] = torch.where(ignored, IGNORED, y)
        # the mean's gradient, tokens weighted a little differently
        weight = 0.5 + torch.rand(t, generator=gen, device="cuda")
        s["g"] = weight / (~ignored).sum().clamp(min=1)
        return s
    n, r, c = case["count"], case["rows"], case["cols"]
    if case["op"] == "orthogonalise":
        s["u"] = _update(n, r, c, _gen(seed, 2)).to(TYPES[case["type"]])
        return s
    s["x"] = torch.randn(n, r, c, generator=_gen(seed, 3), device="cuda").mul_(0.02)
    s["m"] = _update(n, r, c, _gen(seed, 4))
    s["g"] = _update(n, r, c, _gen(seed, 5)).to(TYPES[case["type"]])
    return s


# --------------------------------------------------------------------------------------------------------------------
# the operators


def run(state):
    return (_own if own else _plain)(state, state["case"])


def _own(s, case):
    from paper_1802_04434_b200 import loss, orthogonal
    if case["op"] == "loss":
        return loss.cross_entropy_forward(s["h"], s["w"], s["y"], ignore_index=IGNORED)[0]
    if case["op"] == "train":
        losses, kept = loss.cross_entropy_forward(s["h"], s["w"], s["y"], ignore_index=IGNORED)
        dh, dw = loss.cross_entropy_backward(kept, s["g"])
        return {"losses": losses, "dh": dh, "dw": dw}
    if case["op"] == "orthogonalise":
        return orthogonal.orthogonalise(s["u"], steps=STEPS, coefficients=COEFFICIENTS, dtype=TYPES[case["out"]])
    orthogonal.momentum_step(s["x"], s["g"], s["m"], BETA, DELTA, steps=STEPS, coefficients=COEFFICIENTS, nesterov=case["ahead"])
    return {"x": s["x"], "m": s["m"]}


def _plain(s, case):
    if case["op"] in ("loss", "train"):
        h, w, y, t = s["h"].float(), s["w"].float(), s["y"], TYPES[case["type"]]
        valid = y != IGNORED
        at = torch.where(valid, y, 0)[:, None]
        z = torch.matmul(h, w.t())
        top = z.amax(1, keepdim=True)
        picked = z.gather(1, at)
        e = z.sub_(top).exp_()
        total = e.sum(1, keepdim=True)
        losses = torch.where(valid, (total.log() + (top - picked))[:, 0], 0.0)
        if case["op"] == "loss":
            return losses
        g = torch.where(valid, s["g"], 0.0)[:, None]
        dz = e.mul_(1.0 / total)
        dz.scatter_(1, at, dz.gather(1, at) - 1.0)
        dz.mul_(g)
        return {"losses": losses, "dh": torch.matmul(dz, w).to(t), "dw": torch.matmul(dz.t(), h).to(t)}
    if case["op"] == "orthogonalise":
        return _plain_orthogonal(s["u"].float()).to(TYPES[case["out"]])
    x, m, g = s["x"], s["m"], s["g"].float()
    m.mul_(BETA).add_(g, alpha=1.0 - BETA)
    u = BETA * m + (1.0 - BETA) * g if case["ahead"] else m
    x.sub_(_plain_orthogonal(u), alpha=DELTA)
    return {"x": x, "m": m}


def _plain_orthogonal(u):
    a, b, c = COEFFICIENTS
    tall = u.shape[-2] > u.shape[-1]
    x = u.transpose(-1, -2) if tall else u
    x = x / x.square().sum((-1, -2), keepdim=True).sqrt()
    for _ in range(STEPS):
        g = torch.matmul(x, x.transpose(-1, -2))
        x = a * x + torch.matmul(b * g + c * torch.matmul(g, g), x)
    return x.transpose(-1, -2).contiguous() if tall else x


# --------------------------------------------------------------------------------------------------------------------
# the same in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("loss", "train"):
        return _exact_loss(s, case)
    if case["op"] == "orthogonalise":
        return torch.stack([_exact_orthogonal(u.double()) for u in s["u"]])
    m = 0.95 * s["m"].double() + (1.0 - 0.95) * s["g"].double()
    u = 0.95 * m + (1.0 - 0.95) * s["g"].double() if case["ahead"] else m
    return {"x": torch.stack([x.double() - 0.02 * _exact_orthogonal(v) for x, v in zip(s["x"], u)]), "m": m}


def _exact_loss(s, case):
    """By blocks of tokens: log of the sum of exponentials of the logits' distances from the target's."""
    tokens, width = s["h"].shape
    w, y = s["w"].double(), s["y"]
    losses = torch.zeros(tokens, dtype=torch.float64, device="cuda")
    dh = torch.zeros(tokens, width, dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w)
    for rows in torch.arange(tokens, device="cuda").split(max(1, 100_000_000 // w.shape[0])):
        rows = rows[y[rows] != IGNORED]
        if rows.numel() == 0:
            continue
        h = s["h"][rows].double()
        logits = h @ w.t()
        one = torch.zeros_like(logits)
        one[torch.arange(rows.numel(), device="cuda"), y[rows]] = 1.0
        log_p = torch.log_softmax(logits, 1)
        losses[rows] = -(log_p * one).sum(1)
        if case["op"] == "train":
            d = (log_p.exp() - one) * s["g"][rows].double()[:, None]
            dh[rows] = d @ w
            dw += d.t() @ h
    return losses if case["op"] == "loss" else {"losses": losses, "dh": dh, "dw": dw}


def _exact_orthogonal(u):
    """Through the smaller Gram matrix from the other side: X p(X^T X), p(t) = a + b t + c t^2."""
    if u.shape[0] < u.shape[1]:
        return _exact_orthogonal(u.t()).t()
    x = u / torch.linalg.vector_norm(u)
    one = torch.eye(u.shape[1], dtype=torch.float64, device="cuda")
    for _ in range(5):
        t = x.t() @ x
        x = x @ (3.4445 * one + t @ (-4.7750 * one + 2.0315 * t))
    return x
