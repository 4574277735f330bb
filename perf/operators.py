"""The cases that the language-model operators are measured on, and the operators' plain forms.

Five calls: layer norm and its backward pass, softmax cross entropy of a linear head over a large vocabulary and its
backward pass, and the orthogonalisation of matrix updates by Newton-Schulz products.  ``run`` makes the plain form of a
call (elementary torch operations in 32 bits, rounded once at the end), or with ``own`` the call of
``paper_2210_07454_b200.operators``; ``exact`` gives the definition's value in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5                              # layer norm
STEPS = 5                               # Newton-Schulz
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
BETA = 0.95                             # momentum of the orthogonalised update
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # one row for each of a few sequences in a single-token step, GPT-2-small's width: a call that is all latency
        dict(name="norm_small", op="norm", rows=16, cols=768, dtype="bfloat16"),
        # the rows of a large training batch at a width of 4096
        dict(name="norm_large", op="norm", rows=32768, cols=4096, dtype="bfloat16"),
        # 32-bit training at an odd width and an odd number of rows: nothing is aligned
        dict(name="norm_backward_odd", op="norm_backward", rows=1023, cols=1001, dtype="float32"),
        # 16 sequences of 1024 tokens, GPT-2-small's width
        dict(name="norm_backward_batch", op="norm_backward", rows=16384, cols=768, dtype="bfloat16"),
        # scoring eight tokens with GPT-2-small's vocabulary: the matrix is read once, little is computed
        dict(name="head_tokens", op="head", tokens=8, vocab=50257, width=768, dtype="bfloat16"),
        # the loss of eight sequences of 1024 tokens, same head
        dict(name="head_batch", op="head", tokens=8192, vocab=50257, width=768, dtype="bfloat16"),
        # ragged sizes in fp16: tokens, vocabulary and width end inside every tile
        dict(name="head_backward_odd", op="head_backward", tokens=1000, vocab=32003, width=1000, dtype="float16"),
        # the training step that belongs to head_batch
        dict(name="head_backward_batch", op="head_backward", tokens=8192, vocab=50257, width=768, dtype="bfloat16"),
        # a wide model with a large vocabulary
        dict(name="head_backward_wide", op="head_backward", tokens=4096, vocab=128000, width=4096, dtype="bfloat16"),
        # one small matrix, of odd sizes: fifteen products that depend on one another
        dict(name="orthogonal_small", op="orthogonal", batch=1, rows=100, cols=130, dtype="float32", momentum=False),
        # one matrix of each of GPT-2-small's twelve layers, with its momentum
        dict(name="orthogonal_layers", op="orthogonal", batch=12, rows=768, cols=768, dtype="bfloat16", momentum=True),
        # a matrix of a wide model
        dict(name="orthogonal_wide", op="orthogonal", batch=1, rows=8192, cols=4096, dtype="bfloat16", momentum=False),
    ]


def _spread(rng, low, high):
    """A whole number between the two, spread over its logarithm; even and odd ones alike, a multiple of 64 now and then."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if v > 128 and rng.random() < 0.4:
        v = v // 64 * 64
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "head", "head_backward", "orthogonal"])
    if op.startswith("norm"):
        cols = _spread(rng, 64, 8192)
        rows = _spread(rng, 1, min(65536, 32768 * 4096 // cols))
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["float32", "bfloat16", "float16"]))
    if op.startswith("head"):
        width = _spread(rng, 64, 4096)
        vocab = _spread(rng, 1000, 128000)
        tokens = _spread(rng, 1, 8192)
        return dict(op=op, tokens=tokens if tokens * vocab * width <= 4096 * 128000 * 4096 else 4096, vocab=vocab, width=width,
                    dtype=rng.choice(["bfloat16", "float16"]))
    rows, cols = _spread(rng, 16, 4096), _spread(rng, 16, 4096)
    batch = _spread(rng, 1, max(1, min(16, 8192 * 4096 // (rows * cols))))
    return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=rng.choice(["float32", "bfloat16", "float16"]),
                momentum=rng.random() < 0.5)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    dtype, op = TYPES[case["dtype"]], case["op"]
    state = dict(case=case)
    if op.startswith("norm"):
        # activations with a mean of their own in every row; weights around one
        rows, cols = case["rows"], case["cols"]
        state["x"] = (normal(rows, cols) * 1.5 + normal(rows, 1) * 0.5).to(dtype)
        state["weight"] = 1 + 0.1 * normal(cols)
        state["bias"] = 0.1 * normal(cols)
        if op == "norm_backward":
            state["dy"] = (normal(rows, cols) * 1e-2).to(dtype)
            x = state["x"].float()                                  # what the forward pass keeps
            state["mean"] = x.sum(1) / cols
            centred = x - state["mean"][:, None]
            state["rstd"] = torch.rsqrt((centred * centred).sum(1) / cols + EPS)
    elif op.startswith("head"):
        # normalised hidden states; half of the tokens are predicted with some confidence; one in sixteen is ignored
        tokens, vocab, width = case["tokens"], case["vocab"], case["width"]
        weight = normal(vocab, width) * (2 / math.sqrt(width))
        targets = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
        sure = torch.rand(tokens, generator=gen, device="cuda") < 0.5
        state["hidden"] = (normal(tokens, width) + 2.5 * sure[:, None] * weight[targets]).to(dtype)
        state["weight"] = weight.to(dtype)
        ignored = torch.rand(tokens, generator=gen, device="cuda") < 1 / 16
        ignored[0] = False
        state["targets"] = torch.where(ignored, -100, targets)
        if op == "head_backward":
            state["dloss"] = (0.5 + torch.rand(tokens, generator=gen, device="cuda")) / tokens
            logits = state["hidden"].float() @ state["weight"].float().T    # what the forward pass keeps
            state["lse"] = torch.logsumexp(logits, 1)
    else:
        # gradients of matrices: a few strong directions over noise, as sums of outer products over tokens are
        batch, rows, cols = case["batch"], case["rows"], case["cols"]
        strong = normal(batch, rows, 16) @ normal(batch, 16, cols) / 4
        state["update"] = ((strong + 0.25 * normal(batch, rows, cols)) * 1e-3).to(dtype)
        if case["momentum"]:
            state["momentum"] = (normal(batch, rows, 16) @ normal(batch, 16, cols) / 4 + 0.1 * normal(batch, rows, cols)) * 5e-3
    return state


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2210_07454_b200 import operators
        if op == "norm":
            return operators.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS)
        if op == "norm_backward":
            return operators.layer_norm_backward(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
        if op == "head":
            return operators.linear_cross_entropy(state["hidden"], state["weight"], state["targets"])
        if op == "head_backward":
            return operators.linear_cross_entropy_backward(state["dloss"], state["hidden"], state["weight"], state["targets"],
                                                           state["lse"])
        if "momentum" in state:
            out = operators.orthogonalize(state["update"], momentum=state["momentum"], beta=BETA, nesterov=True, steps=STEPS,
                                          coefficients=COEFFICIENTS)
            return out, state["momentum"]
        return operators.orthogonalize(state["update"], steps=STEPS, coefficients=COEFFICIENTS)
    if op == "norm":
        return _norm(state["x"], state["weight"], state["bias"])
    if op == "norm_backward":
        return _norm_backward(state["dy"], state["x"], state["weight"], state["mean"], state["rstd"])
    if op == "head":
        return _head(state["hidden"], state["weight"], state["targets"])
    if op == "head_backward":
        return _head_backward(state["dloss"], state["hidden"], state["weight"], state["targets"], state["lse"])
    return _orthogonalize(state["update"], state.get("momentum"))


def _norm(x, weight, bias):
    cols, xf = x.shape[1], x.float()
    mean = xf.sum(1) / cols
    centred = xf - mean[:, None]
    rstd = torch.rsqrt((centred * centred).sum(1) / cols + EPS)
    y = centred * rstd[:, None] * weight + bias
    return y.to(x.dtype), mean, rstd


def _norm_backward(dy, x, weight, mean, rstd):
    cols, dyf = x.shape[1], dy.float()
    xhat = (x.float() - mean[:, None]) * rstd[:, None]
    g = dyf * weight
    dx = rstd[:, None] * (g - g.sum(1, keepdim=True) / cols - xhat * ((g * xhat).sum(1, keepdim=True) / cols))
    return dx.to(x.dtype), (dyf * xhat).sum(0), dyf.sum(0)


def _head(hidden, weight, targets):
    logits = hidden.float() @ weight.float().T
    top = logits.amax(1)
    lse = top + torch.log(torch.exp(logits - top[:, None]).sum(1))
    at_target = logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    return torch.where(targets >= 0, lse - at_target, 0.0), lse


def _head_backward(dloss, hidden, weight, targets, lse):
    h, w = hidden.float(), weight.float()
    g = torch.exp(h @ w.T - lse[:, None])
    g.scatter_add_(1, targets.clamp(min=0)[:, None], torch.full_like(lse, -1.0)[:, None])
    g *= torch.where(targets >= 0, dloss, 0.0)[:, None]
    return (g @ w).to(hidden.dtype), (g.T @ h).to(weight.dtype)


def _orthogonalize(update, momentum):
    u = update.float()
    if momentum is not None:
        momentum.mul_(BETA).add_(u)
        u = u + BETA * momentum
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + 1e-7)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    x = x.transpose(1, 2) if tall else x
    out = x.to(torch.float16 if update.dtype == torch.float16 else torch.bfloat16).contiguous()
    return (out, momentum) if momentum is not None else out


def work(case):
    op = case["op"]
    size = 4 if case["dtype"] == "float32" else 2
    if op.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        if op == "norm":
            return {"bytes": 2 * rows * cols * size + 8 * cols + 8 * rows, "flops": 8 * rows * cols}
        return {"bytes": 3 * rows * cols * size + 12 * cols + 8 * rows, "flops": 14 * rows * cols}
    if op.startswith("head"):
        tokens, vocab, width = case["tokens"], case["vocab"], case["width"]
        once = size * (tokens + vocab) * width
        if op == "head":
            return {"bytes": once + 16 * tokens, "flops": 2 * tokens * vocab * width}
        return {"bytes": 2 * once + 16 * tokens, "flops": 6 * tokens * vocab * width}
    batch, rows, cols = case["batch"], case["rows"], case["cols"]
    m, n = min(rows, cols), max(rows, cols)
    # a step: the gram matrix and its square, of which half is enough, and the product with the matrix
    flops = STEPS * batch * (m * m * n + m * m * m + 2 * m * m * n)
    return {"bytes": batch * m * n * (size + 2 + (8 if case["momentum"] else 0)), "flops": flops}


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        x = state["x"].double()
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        return ((x - mean[:, None]) * rstd[:, None]) * state["weight"].double() + state["bias"].double(), mean, rstd
    if op == "norm_backward":
        x, dy, w = state["x"].double(), state["dy"].double(), state["weight"].double()
        mean, rstd = state["mean"].double(), state["rstd"].double()
        h = torch.einsum("rc,r->rc", x - mean[:, None], rstd)
        g = dy * w
        along = torch.einsum("rc,rc->r", g, h) / x.shape[1]
        dx = torch.einsum("rc,r->rc", g - g.mean(1, keepdim=True) - h * along[:, None], rstd)
        return dx, torch.einsum("rc,rc->c", dy, h), dy.sum(0)
    if op.startswith("head"):
        w = state["weight"].double()
        losses, sums, dhs, dw = [], [], [], torch.zeros_like(w)
        for at in range(0, case["tokens"], 1024):                   # rows in pieces: 64-bit logits are large
            part = slice(at, at + 1024)
            h, t = state["hidden"][part].double(), state["targets"][part]
            z = torch.einsum("td,vd->tv", h, w)
            if op == "head":
                sums.append(torch.logsumexp(z, 1))
                picked = torch.einsum("td,td->t", h, w[t.clamp(min=0)])
                losses.append((sums[-1] - picked).masked_fill(t < 0, 0.0))
                continue
            p = z.sub_(state["lse"][part].double()[:, None]).exp_()
            live = (t >= 0).nonzero()[:, 0]
            p[live, t[live]] -= 1.0
            p *= (state["dloss"][part].double() * (t >= 0))[:, None]
            dhs.append(torch.einsum("tv,vd->td", p, w))
            dw += torch.einsum("tv,td->vd", p, h)
        return (torch.cat(losses), torch.cat(sums)) if op == "head" else (torch.cat(dhs), dw)
    u = state["update"].double()
    momentum = None
    if case["momentum"]:
        momentum = BETA * state["momentum"].double() + u
        u = u + BETA * momentum
    x = u / (torch.linalg.matrix_norm(u)[:, None, None] + 1e-7)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):                                          # from the side that is shorter, without forming the square
        if x.shape[1] <= x.shape[2]:
            once = torch.bmm(torch.bmm(x, x.mT), x)
            twice = torch.bmm(torch.bmm(x, x.mT), once)
        else:
            once = torch.bmm(x, torch.bmm(x.mT, x))
            twice = torch.bmm(once, torch.bmm(x.mT, x))
        x = a * x + b * once + c * twice
    return (x, momentum) if momentum is not None else x
