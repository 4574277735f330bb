"""The cases that the operators for experts, dropout and policy tuning are measured on, and the operators' plain forms.

Four operators: the order of tokens by expert, the products of a layer of experts over groups of rows of any size with their gradients,
dropout whose mask is recomputed from a counter and never stored, and the clipped policy loss with its gradient.  ``run`` makes the
plain form of a call (elementary torch operations, rounded once at the end), or with ``own`` the call of
``paper_2210_07454_b200.operators``; ``exact`` gives the definition's value in 64 bits.
"""
import math

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
CLIP = (0.2, 0.28)                      # the policy's ratio stays in 0.8 .. 1.28
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB      # splitmix64
MASK = (1 << 64) - 1


def listed():
    return [
        # eight tokens of a single-token step, two of eight experts each: all latency
        dict(name="sort_step", op="sort", n=16, groups=8),
        # a large batch, 32768 tokens with eight of 256 experts each
        dict(name="sort_batch", op="sort", n=262144, groups=256),
        # the same eight tokens through their experts, GPT-2-small's width: little more than reading the matrices that have a row
        dict(name="grouped_step", op="grouped", rows=16, groups=8, width=768, out=2048, dtype="bfloat16"),
        # 8192 tokens, two of 32 experts each, same width: the training batch of the head
        dict(name="grouped_batch", op="grouped", rows=16384, groups=32, width=768, out=2048, dtype="bfloat16"),
        # ragged in every direction: nothing ends with a tile
        dict(name="grouped_odd", op="grouped", rows=5001, groups=13, width=1001, out=1500, dtype="float16"),
        # the training step that belongs to grouped_batch
        dict(name="grouped_backward_batch", op="grouped_backward", rows=16384, groups=32, width=768, out=2048, dtype="bfloat16"),
        # a wide model with 16 large experts
        dict(name="grouped_backward_wide", op="grouped_backward", rows=16384, groups=16, width=4096, out=2048, dtype="bfloat16"),
        # a few sequences' rows in a small step
        dict(name="dropout_small", op="dropout", rows=16, cols=768, dtype="bfloat16", p=0.1, residual=True),
        # the rows of a large training batch at a width of 4096, added to the residual stream
        dict(name="dropout_batch", op="dropout", rows=32768, cols=4096, dtype="bfloat16", p=0.1, residual=True),
        # the way back in 32 bits, odd sizes
        dict(name="dropout_backward_odd", op="dropout_backward", rows=1023, cols=1001, dtype="float32", p=0.25, residual=False),
        # eight short answers, every sequence of the same weight, with a reference policy; loss and gradient
        dict(name="policy_small", op="policy", tokens=1003, sequences=8, average="sequences", advantage_of="sequences", kl=0.04, masked=True),
        # 512 answers of a large rollout, every token of the same weight; loss and gradient
        dict(name="policy_batch", op="policy", tokens=1000003, sequences=512, average="tokens", advantage_of="tokens", kl=0.01, masked=True),
    ]


def _spread(rng, low, high):
    """A whole number between the two, spread over its logarithm; even and odd ones alike, a multiple of 64 now and then."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if v > 128 and rng.random() < 0.4:
        v = v // 64 * 64
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["sort", "grouped", "grouped", "grouped_backward", "grouped_backward", "dropout", "dropout_backward", "policy"])
    if op == "sort":
        return dict(op=op, n=_spread(rng, 1, 262144), groups=_spread(rng, 1, 512))
    if op.startswith("grouped"):
        width, out = _spread(rng, 64, 4096), _spread(rng, 64, 4096)
        groups = _spread(rng, 1, min(128, (1 << 29) // (width * out)))
        rows = _spread(rng, 1, min(32768, 16384 * 4096 * 2048 // (width * out)))
        return dict(op=op, rows=rows, groups=groups, width=width, out=out, dtype=rng.choice(["bfloat16", "float16"]))
    if op.startswith("dropout"):
        cols = _spread(rng, 64, 8192)
        return dict(op=op, rows=_spread(rng, 1, 32768 * 4096 // cols), cols=cols, dtype=rng.choice(["float32", "bfloat16", "float16"]),
                    p=rng.choice([0.05, 0.1, 0.2, 0.5]), residual=op == "dropout" and rng.random() < 0.7)
    tokens = _spread(rng, 1, 1000003)
    return dict(op=op, tokens=tokens, sequences=_spread(rng, 1, min(2048, tokens)), average=rng.choice(["tokens", "sequences"]),
                advantage_of=rng.choice(["tokens", "sequences"]), kl=rng.choice([0.0, 0.01, 0.1]), masked=rng.random() < 0.7)


def _assignments(n, groups, gen):
    """Experts of n assignments: some experts are asked for more often than others."""
    liking = torch.exp(0.5 * torch.randn(groups, generator=gen, device="cuda"))
    edges = torch.cumsum(liking / liking.sum(), 0)
    return torch.searchsorted(edges, torch.rand(n, generator=gen, device="cuda")).clamp(max=groups - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    op = case["op"]
    state = dict(case=case)
    if op == "sort":
        experts = _assignments(case["n"], case["groups"], gen)
        dropped = torch.rand(case["n"], generator=gen, device="cuda") < 1 / 64      # assignments that were given up: padding, or a full expert
        state["experts"] = torch.where(dropped, -1, experts)
    elif op.startswith("grouped"):
        rows, groups, width, out, dtype = case["rows"], case["groups"], case["width"], case["out"], TYPES[case["dtype"]]
        sizes = torch.bincount(_assignments(rows, groups, gen), minlength=groups)
        state["offsets"] = torch.zeros(groups + 1, dtype=torch.int64, device="cuda")
        state["offsets"][1:] = torch.cumsum(sizes, 0)
        state["ends"] = state["offsets"].tolist()                   # the plain form's loop is the host's
        state["x"] = normal(rows, width).to(dtype)
        state["weight"] = (normal(groups, out, width) / math.sqrt(width)).to(dtype)
        if op == "grouped_backward":
            state["dy"] = (normal(rows, out) * 1e-2).to(dtype)
    elif op.startswith("dropout"):
        rows, cols, dtype = case["rows"], case["cols"], TYPES[case["dtype"]]
        state["seed"] = (seed * GAMMA + 12345) & MASK
        state["x"] = normal(rows, cols).to(dtype)
        if case["residual"]:
            state["residual"] = (2 * normal(rows, cols)).to(dtype)
    else:
        tokens, sequences = case["tokens"], case["sequences"]
        cuts = torch.sort(torch.randint(0, tokens + 1, (sequences - 1,), generator=gen, device="cuda")).values
        state["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), tokens)])
        # losses of a trained model's own samples; the policy has moved a little since, further from its reference
        state["old_nll"] = -torch.log(torch.rand(tokens, generator=gen, device="cuda").clamp(min=1e-6)) * 0.8
        state["nll"] = (state["old_nll"] + 0.15 * normal(tokens)).clamp(min=0)
        state["reference_nll"] = (state["old_nll"] + 0.4 * normal(tokens)).clamp(min=0) if case["kl"] else None
        state["advantages"] = normal(tokens if case["advantage_of"] == "tokens" else sequences)
        state["targets"] = None
        if case["masked"]:                                           # prompts and padding take no part
            targets = torch.randint(0, 50257, (tokens,), generator=gen, device="cuda")
            state["targets"] = torch.where(torch.rand(tokens, generator=gen, device="cuda") < 0.25, -100, targets)
        state["dloss"] = torch.full((1,), 0.5, device="cuda")
    return state


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2210_07454_b200 import operators
        if op == "sort":
            return operators.sort_by_expert(state["experts"], case["groups"])
        if op == "grouped":
            return operators.grouped_linear(state["x"], state["weight"], state["offsets"])
        if op == "grouped_backward":
            return operators.grouped_linear_backward(state["dy"], state["x"], state["weight"], state["offsets"])
        if op == "dropout":
            return operators.dropout(state["x"], case["p"], state["seed"], residual=state.get("residual"))
        if op == "dropout_backward":
            return operators.dropout_backward(state["x"], case["p"], state["seed"])
        common = dict(targets=state["targets"], offsets=state["offsets"], reference_nll=state["reference_nll"], clip=CLIP, kl=case["kl"],
                      advantage_of=case["advantage_of"])
        result, norm = operators.policy_loss(state["nll"], state["old_nll"], state["advantages"], average=case["average"], **common)
        return result, norm, operators.policy_loss_backward(state["dloss"], state["nll"], state["old_nll"], state["advantages"], norm, **common)
    if op == "sort":
        return _sort(state["experts"], case["groups"])
    if op == "grouped":
        return _grouped(state["x"], state["weight"], state["ends"])
    if op == "grouped_backward":
        return _grouped_backward(state["dy"], state["x"], state["weight"], state["ends"])
    if op.startswith("dropout"):
        return _dropout(state["x"], case["p"], state["seed"], state.get("residual"))
    return _policy(state, case)


def _sort(experts, groups):
    key = torch.where((experts >= 0) & (experts < groups), experts, groups)
    order = torch.argsort(key, stable=True)
    places = torch.empty_like(order)
    places[order] = torch.arange(len(order), device=order.device)
    sizes = (key[:, None] == torch.arange(groups, device=key.device)).sum(0)
    offsets = torch.zeros(groups + 1, dtype=torch.int64, device=key.device)
    offsets[1:] = torch.cumsum(sizes, 0)
    return order, places, offsets


def _grouped(x, weight, ends):
    y = torch.zeros(x.shape[0], weight.shape[1], device=x.device)
    for g in range(weight.shape[0]):
        if ends[g + 1] > ends[g]:
            y[ends[g]:ends[g + 1]] = x[ends[g]:ends[g + 1]].float() @ weight[g].float().T
    return y.to(x.dtype)


def _grouped_backward(dy, x, weight, ends):
    dx = torch.zeros(x.shape, device=x.device)
    dweight = torch.zeros(weight.shape, device=x.device)
    for g in range(weight.shape[0]):
        if ends[g + 1] > ends[g]:
            part = slice(ends[g], ends[g + 1])
            d = dy[part].float()
            dx[part] = d @ weight[g].float()
            dweight[g] = d.T @ x[part].float()
    return dx.to(x.dtype), dweight.to(weight.dtype)


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _shifted(z, by):
    return (z >> by) & ((1 << (64 - by)) - 1)                       # 64-bit whole numbers of torch are signed


def _kept(n, p, seed, device):
    """Which of n values stay, and by what they are multiplied."""
    z = (seed + GAMMA) & MASK                                       # the key: the first output of the stream that starts at the seed
    z = (z ^ (z >> 30)) * MIX1 & MASK
    z = (z ^ (z >> 27)) * MIX2 & MASK
    key = z ^ (z >> 31)
    z = torch.arange(1, (n + 3) // 4 + 1, device=device) * _signed(GAMMA) + _signed(key)
    z = (z ^ _shifted(z, 30)) * _signed(MIX1)
    z = (z ^ _shifted(z, 27)) * _signed(MIX2)
    z = z ^ _shifted(z, 31)
    below = round(p * 65536)
    fields = torch.stack([_shifted(z, 16 * i) & 0xFFFF if i else z & 0xFFFF for i in range(4)], 1)
    return (fields >= below).view(-1)[:n], 65536 / (65536 - below)


def _dropout(x, p, seed, residual):
    keep, scale = _kept(x.numel(), p, seed, x.device)
    y = torch.where(keep.view(x.shape), x.float() * scale, 0.0)
    if residual is not None:
        y = y + residual.float()
    return y.to(x.dtype)


def _policy(state, case):
    nll, old, advantages, offsets, targets = state["nll"], state["old_nll"], state["advantages"], state["offsets"], state["targets"]
    sequences = len(offsets) - 1
    sequence = torch.searchsorted(offsets[1:], torch.arange(len(nll), device=nll.device), right=True)
    live = targets >= 0 if targets is not None else torch.ones_like(nll, dtype=torch.bool)
    if case["advantage_of"] == "sequences":
        advantages = advantages[sequence]
    d = old.double() - nll.double()                                 # 64 bits: what is clipped is decided on it
    ratio = torch.exp(d.float())
    up = advantages >= 0
    clipped = torch.where(up, d > math.log1p(CLIP[1]), d < math.log1p(-CLIP[0]))
    held = torch.where(up, 1 + CLIP[1], 1 - CLIP[0])
    loss = -advantages * torch.where(clipped, held, ratio)
    slope = torch.where(clipped, 0.0, advantages * ratio)
    kl = torch.zeros_like(nll)
    if state["reference_nll"] is not None:
        e = nll.double() - state["reference_nll"].double()
        kl = (torch.exp(e) - e - 1).float()                         # 64 bits: near 0 the three cancel
        loss = loss + case["kl"] * kl
        slope = slope + case["kl"] * (torch.exp(e) - 1).float()
    counts = torch.zeros(sequences, dtype=torch.float64, device=nll.device).index_add_(0, sequence, live.double())
    if case["average"] == "tokens":
        norm = torch.where(counts.sum() > 0, 1 / counts.sum(), 0.0).expand(sequences)
    else:
        norm = torch.where(counts > 0, 1 / (counts * (counts > 0).sum()), 0.0)
    weight = torch.where(live, norm[sequence], 0.0)                 # a long sum: in 64 bits
    result = torch.stack([(weight * v).sum() for v in (loss, kl, clipped)])
    return result.float(), norm.float(), state["dloss"] * weight.float() * slope


def work(case):
    op = case["op"]
    if op == "sort":
        return {"bytes": 24 * case["n"] + 8 * case["groups"], "flops": case["n"]}
    if op.startswith("grouped"):
        rows, groups, width, out = case["rows"], case["groups"], case["width"], case["out"]
        live = groups * (1 - (1 - 1 / groups) ** rows)              # experts that have a row
        if op == "grouped":
            return {"bytes": int(2 * (rows * (width + out) + live * width * out)), "flops": 2 * rows * width * out}
        return {"bytes": int(2 * (rows * (2 * width + out) + (live + groups) * width * out)), "flops": 4 * rows * width * out}
    if op.startswith("dropout"):
        n = case["rows"] * case["cols"]
        return {"bytes": n * (4 if case["dtype"] == "float32" else 2) * (3 if case["residual"] else 2), "flops": 2 * n}
    tokens, sequences = case["tokens"], case["sequences"]
    a_token = 12 + (4 if case["kl"] else 0) + (8 if case["masked"] else 0) + (4 if case["advantage_of"] == "tokens" else 0)
    return {"bytes": tokens * a_token + sequences * (16 if case["advantage_of"] == "sequences" else 12), "flops": 20 * tokens}


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "sort":
        n, groups = case["n"], case["groups"]
        e = state["experts"]
        e = e + (e < 0) * (groups - e)                              # the given-up ones behind the last expert
        pairs = torch.sort(e * n + torch.arange(n, device=e.device)).values
        order = pairs % n
        places = torch.zeros_like(order).scatter_(0, order, torch.arange(n, device=e.device))
        return order, places, torch.searchsorted(pairs, torch.arange(groups + 1, device=e.device) * n)
    if op.startswith("grouped"):
        x, ends = state["x"], state["offsets"].tolist()
        pieces, dweight = [], []
        for w, a, b in zip(state["weight"], ends, ends[1:]):
            w = w.double()
            if op == "grouped":
                pieces.append(torch.einsum("rk,nk->rn", x[a:b].double(), w))
                continue
            d = state["dy"][a:b].double()
            pieces.append(torch.einsum("rn,nk->rk", d, w))
            dweight.append(torch.einsum("rn,rk->nk", d, x[a:b].double()))
        return torch.cat(pieces) if op == "grouped" else (torch.cat(pieces), torch.stack(dweight))
    if op.startswith("dropout"):
        x = state["x"]
        n = x.numel()
        # the generator in 32-bit halves of unsigned numbers, so that no product passes 63 bits
        low, high = _split(state["seed"], GAMMA, torch.ones(1, dtype=torch.int64, device=x.device))
        key = int(high[0]) << 32 | int(low[0])
        low, high = _split(key, GAMMA, torch.arange(1, (n + 3) // 4 + 1, device=x.device))
        quarter = torch.stack([low % 65536, low // 65536, high % 65536, high // 65536], -1).flatten()[:n].view(x.shape)
        below = int(math.floor(case["p"] * 65536 + 0.5))
        y = x.double() * (quarter >= below) / (1 - below / 65536)
        return y + state["residual"].double() if case["residual"] else y
    nll, old, a = state["nll"].double(), state["old_nll"].double(), state["advantages"].double()
    lengths = state["offsets"].diff()
    number = torch.repeat_interleave(torch.arange(len(lengths), device=nll.device), lengths)
    if case["advantage_of"] == "sequences":
        a = a[number]
    live = (state["targets"] >= 0).double() if case["masked"] else torch.ones_like(nll)
    r = (old - nll).exp()
    objective = torch.minimum(r * a, r.clamp(1 - CLIP[0], 1 + CLIP[1]) * a)
    cut = ((a >= 0) & (r > 1 + CLIP[1])) | ((a < 0) & (r < 1 - CLIP[0]))
    gradient = (a * r).masked_fill(cut, 0.0)
    k = torch.zeros_like(nll)
    if case["kl"]:
        e = nll - state["reference_nll"].double()
        k = torch.expm1(e) - e
        gradient = gradient + case["kl"] * torch.expm1(e)
    table = torch.zeros(len(lengths), dtype=torch.float64, device=nll.device).scatter_add_(0, number, live)
    if case["average"] == "tokens":
        norm = torch.full_like(table, 1 / float(table.sum()) if float(table.sum()) else 0.0)
    else:
        norm = (1 / table / (table > 0).sum()).masked_fill(table == 0, 0.0)
    share = live * norm[number]
    result = torch.stack([torch.dot(share, case["kl"] * k - objective), torch.dot(share, k), torch.dot(share, cut.double())])
    return result, norm, share * gradient * float(state["dloss"])


def _product(low, high, c):
    """(low + 2^32 high) c modulo 2^64, in halves"""
    c0, c1, c2 = c & 0xFFFF, c >> 16 & 0xFFFF, c >> 32
    p0, p1 = low * c0, low * c1                                     # below 2^48
    at16 = (p0 >> 16) + p1                                          # what stands from bit 16 on
    new_low = (p0 & 0xFFFF) | (at16 & 0xFFFF) << 16
    c2l, c2h = c2 & 0xFFFF, c2 >> 16
    low_c2 = (low * c2l & 0xFFFFFFFF) + ((low * c2h & 0xFFFF) << 16)
    high_c = high * c0 + ((high * c1 & 0xFFFF) << 16)
    return new_low, ((at16 >> 16) + low_c2 + high_c) & 0xFFFFFFFF


def _xorshift(low, high, by):
    """z ^ (z >> by), by below 32, in halves"""
    return low ^ ((low >> by) | (high << (32 - by)) & 0xFFFFFFFF), high ^ (high >> by)


def _split(start, gamma, counter):
    """Output number `counter` (1, 2, ...) of splitmix64 begun at `start`, as its low and its high half."""
    low, high = _product(counter & 0xFFFFFFFF, counter >> 32, gamma)
    low = low + (start & 0xFFFFFFFF)
    high = (high + (start >> 32) + (low >> 32)) & 0xFFFFFFFF
    low = low & 0xFFFFFFFF
    low, high = _product(*_xorshift(low, high, 30), MIX1)
    low, high = _product(*_xorshift(low, high, 27), MIX2)
    return _xorshift(low, high, 31)
