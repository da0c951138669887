"""The operators around a plan that are timed, and what they have to give.

Three operators of a mixture-of-experts layer stand next to the planning step:

  router    scores of a token's experts -> the top_k expert ids that a plan starts from, and the
            weights of the chosen experts; forward and backward
  experts   the whole expert layer for a few tokens, on the physical instances a plan names: per
            token the weighted sum of its instances' gated feed-forward networks
  clip      the global norm of many gradient tensors, and their scaling to a largest norm

Every case has a plain form here (elementary torch operations in 32 bits, rounded once at the end)
and a value in 64 bits.  With `own` set, run() makes the calls a user makes of this package.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEVICE = "cuda"
SIGMOID_EPS = 1e-20   # added to the sum of the chosen sigmoid scores before weights are normalised
CLIP_EPS = 1e-6       # added to the norm before the clipping factor is formed


# ---------------------------------------------------------------------------------- the cases

def listed():
    return [
        # decoding: the router of one DeepSeek-V3-shaped layer for the one token of a step
        dict(name="router one token", op="router", way="forward", tokens=1, experts=256, top_k=8,
             dtype="bf16", score="sigmoid", bias=True, normalize=True, scale=2.5),
        # training: the tokens of one rank, scores kept in 32 bits, aux-loss-free balancing bias
        dict(name="router rank", op="router", way="forward", tokens=8192, experts=256, top_k=8,
             dtype="f32", score="sigmoid", bias=True, normalize=True, scale=2.5),
        # training: all 32 ranks' tokens of one layer, as planned on one GPU
        dict(name="router group", op="router", way="forward", tokens=262144, experts=256, top_k=8,
             dtype="f32", score="softmax", bias=False, normalize=True, scale=1.0),
        # training: the gradient of 64 experts' scores (32 ranks x 4096 tokens)
        dict(name="router backward group", op="router", way="backward", tokens=131072, experts=64,
             top_k=6, dtype="bf16", score="softmax", bias=False, normalize=False, scale=1.0),
        # a ragged microbatch of a model whose expert count is no power of two
        dict(name="router backward odd", op="router", way="backward", tokens=1023, experts=60,
             top_k=3, dtype="f32", score="sigmoid", bias=False, normalize=True, scale=1.0),
        # decoding one token with a small layer: latency
        dict(name="experts one token, small", op="experts", tokens=1, top_k=2, ranks=1, e_loc=32,
             slots=0, hidden=1024, ffn=2048, spread=False),
        # decoding a few requests on a mid-sized layer
        dict(name="experts 16 tokens, mid", op="experts", tokens=16, top_k=6, ranks=1, e_loc=64,
             slots=0, hidden=2048, ffn=1408, spread=False),
        # decoding one token with DeepSeek-V3-shaped experts, a node's eight ranks on one GPU
        dict(name="experts one token, large", op="experts", tokens=1, top_k=8, ranks=8, e_loc=8,
             slots=1, hidden=7168, ffn=2048, spread=False),
        # one EP rank of 32: the rows that 32 ranks' requests sent it, most of their ids elsewhere
        dict(name="experts 128 rows of a rank", op="experts", tokens=128, top_k=8, ranks=1,
             e_loc=8, slots=1, hidden=7168, ffn=2048, spread=True),
        # the gradients of one router: a few small tensors, latency
        dict(name="clip a router", op="clip", tensors=3, elements=33000, kinds="f32", clipped=False,
             even=False),
        # a model's small tensors, packed one after the other, of two types
        dict(name="clip 300 ragged tensors", op="clip", tensors=300, elements=24_000_000,
             kinds="bf16,f32", clipped=True, even=False),
        # the three matrices of a rank's eight DeepSeek-V3-shaped experts
        dict(name="clip a rank's experts", op="clip", tensors=24, elements=24 * 7168 * 2048,
             kinds="bf16", clipped=True, even=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["router", "experts", "clip"])
    if op == "router":
        experts = _log(rng, 8, 512)
        score = rng.choice(["softmax", "sigmoid"])
        return dict(op=op, way=rng.choice(["forward", "backward"]), tokens=_log(rng, 1, 100000),
                    experts=experts, top_k=rng.randint(1, min(8, experts)),
                    dtype=rng.choice(["f32", "bf16", "f16"]), score=score,
                    bias=score == "sigmoid" and rng.random() < 0.5,
                    normalize=rng.random() < 0.5, scale=rng.choice([1.0, 2.5]))
    if op == "experts":
        ranks = rng.randint(1, 4)
        e_loc, slots = _log(rng, 1, 24), rng.randint(0, 2)
        return dict(op=op, tokens=_log(rng, 1, 128), top_k=rng.randint(1, min(8, ranks * e_loc)),
                    ranks=ranks, e_loc=e_loc, slots=slots, hidden=8 * _log(rng, 16, 512),
                    ffn=8 * _log(rng, 16, 256), spread=rng.random() < 0.4)
    tensors = _log(rng, 1, 300)
    return dict(op=op, tensors=tensors, elements=max(tensors, _log(rng, 2000, 100_000_000)),
                kinds=rng.choice(["f32", "bf16", "f16", "bf16,f32"]), clipped=rng.random() < 0.7,
                even=rng.random() < 0.3)


# --------------------------------------------------------------------------------- the inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    return {"router": _prepare_router, "experts": _prepare_experts,
            "clip": _prepare_clip}[case["op"]](case, seed)


def _popularity(n, g):
    """Logarithm of a Zipf popularity (exponent 1.1) over a random order of n experts."""
    order = torch.randperm(n, generator=g, device=DEVICE)
    return -1.1 * torch.log(order.float() + 1.0)


def _router_inputs(case, seed):
    """Logits with a fixed part for each expert, a balancing bias, and where the gradient is asked
    for the ids and weights of the forward pass and the weights' gradient."""
    g = _generator(seed)
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    logits = torch.empty(T, E, device=DEVICE).normal_(generator=g)
    logits += 0.5 * _popularity(E, g)
    logits = logits.to(DTYPES[case["dtype"]])
    bias = 0.1 * torch.randn(E, generator=g, device=DEVICE) if case["bias"] else None
    s = dict(logits=logits, bias=bias)
    if case["way"] == "backward":
        s["ids"], s["weights"] = _router_forward(logits, bias, case)
        s["grad_weights"] = torch.randn(T, k, generator=g, device=DEVICE)
    return s


def _prepare_router(case, seed):
    s = dict(_router_inputs(case, seed), case=case)
    if own:
        from paper_2609_35481_b200 import Router
        s["router"] = Router(case["experts"], case["top_k"], score=case["score"],
                             normalize=case["normalize"], scale=case["scale"])
    return s


def _experts_inputs(case, seed):
    """Rows, instance ids and weights of a few tokens, and the parameter blocks of the instances:
    main [ranks][e_loc][|W|] and replica [ranks][slots][|W|] bytes, a block being the gate matrix
    [ffn][hidden], the up matrix [ffn][hidden] and the down matrix [hidden][ffn] in bf16."""
    g = _generator(seed)
    T, k, H, F = case["tokens"], case["top_k"], case["hidden"], case["ffn"]
    R, L, N = case["ranks"], case["e_loc"], case["slots"]
    per = 3 * H * F
    blocks = []
    for n in (R * L, R * N):
        b = torch.empty(n, per, dtype=torch.bfloat16, device=DEVICE).normal_(generator=g)
        b[:, :2 * H * F] *= H ** -0.5
        b[:, 2 * H * F:] *= F ** -0.5
        blocks.append(b.view(torch.uint8).view(R, n // R, 2 * per))
    x = torch.empty(T, H, dtype=torch.bfloat16, device=DEVICE).normal_(generator=g)
    # distinct experts a token; a replica slot stands in for the expert of the same number
    noise = -torch.log(-torch.log(torch.rand(T, R * L, generator=g, device=DEVICE) + 1e-9) + 1e-9)
    expert = torch.topk(_popularity(R * L, g) + noise, min(k, R * L), dim=1).indices
    rank, local = expert // L, expert % L
    away = (local < N) & (torch.rand(expert.shape, generator=g, device=DEVICE) < 0.5)
    ids = rank * (L + N) + torch.where(away, L + local, local)
    ids = torch.nn.functional.pad(ids, (0, k - ids.shape[1]), value=-1)
    if case["spread"]:   # most of a row's ids live on other ranks
        keep = torch.rand(T, k, generator=g, device=DEVICE) < 0.15
        keep[:, 0] = True
        ids = torch.where(keep, ids, -1)
        ids = ids.gather(1, torch.rand(T, k, generator=g, device=DEVICE).argsort(1))
    weights = torch.softmax(torch.randn(T, k, generator=g, device=DEVICE), 1)
    return dict(x=x, ids=ids.to(torch.int32), weights=weights, main=blocks[0],
                replica=blocks[1] if N else None)


def _prepare_experts(case, seed):
    s = dict(_experts_inputs(case, seed), case=case)
    if own:
        from paper_2609_35481_b200 import TokenExperts
        s["layer"] = TokenExperts(case["hidden"], case["ffn"], case["top_k"], case["tokens"],
                                  case["e_loc"], slots_per_rank=case["slots"], ranks=case["ranks"])
        s["layer"].set_experts(s["main"], s["replica"])
    return s


def _clip_inputs(case, seed):
    """Gradient tensors packed one after the other in one buffer for each type, as a training
    program keeps them, and buffers of the same layout for the clipped ones."""
    n, total = case["tensors"], case["elements"]
    if case["even"]:
        sizes = np.full(n, total // n)
    else:   # a few large tensors and many small ones; the sizes belong to the model, not the seed
        share = np.random.default_rng(n).dirichlet(np.full(n, 0.5)) * (total - n)
        sizes = 1 + share.astype(np.int64)
    kinds = _kinds(case)
    g = _generator(seed)
    grads, outs, flats = [None] * n, [None] * n, {}
    for kind in sorted(set(kinds)):
        mine = [i for i in range(n) if kinds[i] == kind]
        src = torch.empty(int(sum(sizes[i] for i in mine)), dtype=DTYPES[kind],
                          device=DEVICE).normal_(std=1e-3, generator=g)
        dst = torch.zeros_like(src)
        at = 0
        for i in mine:
            m = int(sizes[i])
            grads[i], outs[i] = src[at:at + m], dst[at:at + m]
            at += m
        flats[kind] = dst
    expected = 1e-3 * math.sqrt(float(sum(sizes)))
    return dict(grads=grads, outs=outs, flats=flats,
                max_norm=expected * (0.37 if case["clipped"] else 3.0))


def _prepare_clip(case, seed):
    s = dict(_clip_inputs(case, seed), case=case)
    if own:
        from paper_2609_35481_b200 import GradientClip
        s["clip"] = GradientClip(s["grads"], out=s["outs"])
    return s


# ------------------------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if case["op"] == "router":
        if case["way"] == "forward":
            if own:
                ids, weights = s["router"].forward(s["logits"], bias=s["bias"])
            else:
                ids, weights = _router_forward(s["logits"], s["bias"], case)
            return {"ids": ids, "weights": weights}
        if own:
            return s["router"].backward(s["logits"], s["ids"], s["weights"], s["grad_weights"])
        return _router_backward(s["logits"], s["ids"], s["weights"], s["grad_weights"], case)
    if case["op"] == "experts":
        if own:
            return s["layer"].forward(s["x"], s["ids"], s["weights"])
        return _experts_forward(s, case)
    if own:
        norm = s["clip"].clip(s["max_norm"])
    else:
        norm = _clip(s["grads"], s["outs"], s["max_norm"])
    return {"norm": norm, "grads": s["flats"]}


def _router_forward(logits, bias, case):
    """ids in descending order of the choice value, ties to the lowest id.  The choice value is
    the logit, or with a bias the sigmoid score plus the bias; one of -inf or NaN is not chosen."""
    x = logits.float()
    choice = x if bias is None else 1.0 / (1.0 + torch.exp(-x)) + bias
    choice = torch.where(torch.isnan(choice) | (x == -math.inf), -math.inf, choice)
    value, ids = torch.sort(choice, dim=1, descending=True, stable=True)
    value, ids = value[:, :case["top_k"]], ids[:, :case["top_k"]]
    taken = value != -math.inf
    picked = x.gather(1, ids)
    if case["score"] == "sigmoid":
        w = torch.where(taken, 1.0 / (1.0 + torch.exp(-picked)), 0.0)
        if case["normalize"]:
            w = w / (w.sum(1, keepdim=True) + SIGMOID_EPS)
    else:
        top = picked[:, :1]
        w = torch.where(taken, torch.exp(picked - top), 0.0)
        if case["normalize"]:
            w = w / w.sum(1, keepdim=True)
        else:
            w = w / torch.exp(x - top).sum(1, keepdim=True)
    w = torch.where(taken, w * case["scale"], 0.0)
    return torch.where(taken, ids, -1).to(torch.int32), w


def _router_backward(logits, ids, weights, grad_weights, case):
    taken = ids >= 0
    at = torch.where(taken, ids, 0).long()
    w, dw = torch.where(taken, weights, 0.0), torch.where(taken, grad_weights, 0.0)
    mean = (w * dw).sum(1, keepdim=True) / case["scale"]
    part = w * (dw - mean) if case["normalize"] else w * dw
    if case["score"] == "sigmoid":
        part = part / (1.0 + torch.exp(logits.gather(1, at).float()))
        grad = torch.zeros(logits.shape, device=logits.device)
    elif case["normalize"]:
        grad = torch.zeros(logits.shape, device=logits.device)
    else:
        x = logits.float()
        p = torch.exp(x - x.amax(1, keepdim=True))
        grad = -(p / p.sum(1, keepdim=True)) * (mean * case["scale"])
        grad = torch.where(taken.any(1, keepdim=True), grad, 0.0)
    return grad.scatter_add(1, at, part).to(logits.dtype)


def _experts_forward(s, case):
    H, F, T, k = case["hidden"], case["ffn"], case["tokens"], case["top_k"]
    blocks = s["main"] if s["replica"] is None else torch.cat([s["main"], s["replica"]], 1)
    blocks = blocks.reshape(-1, 6 * H * F).view(torch.bfloat16)
    first, down = blocks[:, :2 * H * F].view(-1, 2 * F, H), blocks[:, 2 * H * F:].view(-1, H, F)
    x = s["x"].float()
    y = torch.zeros(T, H, device=x.device)
    for j in range(k):
        here = s["ids"][:, j] >= 0
        e = torch.where(here, s["ids"][:, j], 0).long()
        gu = torch.bmm(first[e].float(), x[:, :, None])[:, :, 0]
        h = gu[:, :F] / (1.0 + torch.exp(-gu[:, :F])) * gu[:, F:]
        out = torch.bmm(down[e].float(), h[:, :, None])[:, :, 0]
        y += torch.where(here[:, None], out * s["weights"][:, j:j + 1], 0.0)
    return y.to(s["x"].dtype)


def _clip(grads, outs, max_norm):
    norm = torch.sqrt(torch.stack([torch.sum(t.float() * t.float()) for t in grads]).sum())
    factor = torch.clamp(max_norm / (norm + CLIP_EPS), max=1.0)
    for t, o in zip(grads, outs):
        o.copy_(t.float() * factor)
    return norm


# ------------------------------------------------------------------------- what cannot be left

def work(case):
    if case["op"] == "router":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        size = 4 if case["dtype"] == "f32" else 2
        if case["way"] == "forward":
            # every logit read, an id and a weight written for each choice
            return {"bytes": T * E * size + 8 * T * k + (4 * E if case["bias"] else 0),
                    "flops": 4 * T * E}
        # every gradient written; id, weight and its gradient read for each choice; the full row of
        # logits only where the softmax over all experts is differentiated
        read = T * E * size if case["score"] == "softmax" and not case["normalize"] else \
            T * k * size if case["score"] == "sigmoid" else 0
        return {"bytes": T * E * size + 12 * T * k + read, "flops": 4 * T * E}
    if case["op"] == "experts":
        # the blocks of the instances that some row names are read once, whatever the rows
        T, k, H, F = case["tokens"], case["top_k"], case["hidden"], case["ffn"]
        chosen = T * k if not case["spread"] else T * (1 + 0.15 * (k - 1))
        distinct = _distinct(case, chosen)
        return {"bytes": distinct * 6 * H * F + 4 * T * H + 8 * T * k,
                "flops": 6 * H * F * chosen}
    sizes = 4 if case["kinds"] == "f32" else 2 if "," not in case["kinds"] else 3
    return {"bytes": 2 * sizes * case["elements"], "flops": 3 * case["elements"]}


def _distinct(case, chosen):
    """Expected number of different instances among `chosen` ids of the Zipf popularity."""
    n = case["ranks"] * case["e_loc"]
    p = np.arange(1, n + 1, dtype=np.float64) ** -1.1
    p /= p.sum()
    per = min(case["top_k"], n) * p
    per = np.minimum(1.0, per * (min(case["top_k"], n) / max(np.minimum(1.0, per).sum(), 1e-9)))
    seen = 1.0 - (1.0 - per) ** (chosen / case["top_k"])
    if case["tokens"] == 1:
        seen = np.full(n, min(case["top_k"], n) / n)
    copies = 1.0 + 0.5 * min(1.0, case["slots"] / case["e_loc"]) * (1 if case["tokens"] > 1 else 0)
    return min(float(seen.sum()) * copies, n + case["ranks"] * case["slots"], chosen)


# ----------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    if case["op"] == "router":
        s = _router_inputs(case, seed)
        return _exact_router(s, case)
    if case["op"] == "experts":
        return _exact_experts(_experts_inputs(case, seed), case)
    return _exact_clip(_clip_inputs(case, seed), case)


def _exact_router(s, case):
    x = s["logits"].double()
    T, E, k, c = case["tokens"], case["experts"], case["top_k"], case["scale"]
    if case["way"] == "forward":
        # which experts are chosen is settled by the 32-bit scores; one maximum after the other
        left = s["logits"].float().clone()
        if s["bias"] is not None:
            left = 1.0 / (1.0 + torch.exp(-left)) + s["bias"]
        number = torch.arange(E, device=x.device)
        ids = torch.empty(T, k, dtype=torch.int64, device=x.device)
        for j in range(k):
            best = left.amax(1, keepdim=True)
            ids[:, j] = torch.where(left == best, number, E).amin(1)
            left.scatter_(1, ids[:, j:j + 1], -math.inf)
        z = x.gather(1, ids)
        if case["score"] == "sigmoid":
            w = torch.special.expit(z)
            if case["normalize"]:
                w = w / (w.sum(1, keepdim=True) + SIGMOID_EPS)
        else:
            w = torch.exp(z - torch.logsumexp(z if case["normalize"] else x, 1, keepdim=True))
        return {"ids": ids.to(torch.int32), "weights": c * w}
    # the gradient through the definition itself, by differentiating the 64-bit weights
    z = x.detach().requires_grad_(True)
    picked = z.gather(1, s["ids"].long())
    if case["score"] == "sigmoid":
        w = torch.special.expit(picked)
        w = w / (w.sum(1, keepdim=True) + SIGMOID_EPS) if case["normalize"] else w
    elif case["normalize"]:
        w = torch.softmax(picked, 1)
    else:
        w = torch.softmax(z, 1).gather(1, s["ids"].long())
    (c * w * s["grad_weights"].double()).sum().backward()
    return z.grad


def _exact_experts(s, case):
    H, F, L, N = case["hidden"], case["ffn"], case["e_loc"], case["slots"]
    x, y = s["x"].double(), torch.zeros(case["tokens"], H, dtype=torch.float64, device=DEVICE)
    for p in sorted(set(s["ids"].flatten().tolist()) - {-1}):
        r, l = divmod(p, L + N)
        block = (s["main"][r, l] if l < L else s["replica"][r, l - L]).view(torch.bfloat16)
        gate, up, down = (block[i * H * F:(i + 1) * H * F].double() for i in range(3))
        t, j = torch.nonzero(s["ids"] == p, as_tuple=True)
        g, u = x[t] @ gate.view(F, H).T, x[t] @ up.view(F, H).T
        h = g * torch.special.expit(g) * u
        y.index_add_(0, t, (h @ down.view(H, F).T) * s["weights"][t, j].double()[:, None])
    return y


def _exact_clip(s, case):
    total = 0.0
    for t in s["grads"]:
        total += float(torch.linalg.vector_norm(t.double())) ** 2
    norm = math.sqrt(total)
    factor = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
    flats = {}
    for t, o, kind in zip(s["grads"], s["outs"], _kinds(case)):
        flats.setdefault(kind, []).append(t.double() * factor)
    return {"norm": torch.tensor(norm, dtype=torch.float64),
            "grads": {kind: torch.cat(v) for kind, v in flats.items()}}


def _kinds(case):
    kinds = case["kinds"].split(",")
    return [kinds[i % len(kinds)] for i in range(case["tensors"])]
