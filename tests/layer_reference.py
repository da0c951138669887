"""Plain 64-bit forms of the layer operators, written from their definitions for the tests, and the
error bounds that the CUDA results are held to."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -24                                      # unit roundoff of 32 bits
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def router_forward(logits, k, score, normalize, scale, bias=None, mask=None):
    """(ids, weights) token by token with Python's own sort; the choice value of a biased sigmoid
    is a 32-bit number by definition."""
    l32 = logits.float().cpu()
    choice = l32 if bias is None else 1.0 / (1.0 + torch.exp(-l32)) + bias.float().cpu()
    T, E = l32.shape
    ids = torch.full((T, k), -1, dtype=torch.int32)
    w = torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        row, c = l32[t].tolist(), choice[t].tolist()
        left = [i for i in range(E) if c[i] > -math.inf and row[i] > -math.inf]
        chosen = sorted(left, key=lambda i: (-c[i], i))[:k]
        if not chosen:
            continue
        z = l32[t].double()
        if score == "sigmoid":
            v = torch.special.expit(z[chosen])
            v = v / (v.sum() + 1e-20) if normalize else v
        else:
            over = z[chosen] if normalize else z
            top = over.max()     # subtracted first: the type's lowest value swallows a log
            v = torch.exp(z[chosen] - top) / torch.exp(over - top).sum()
        ids[t, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
        w[t, :len(chosen)] = scale * v
    return ids, w


def router_forward_many(logits, k, score, normalize, scale, bias=None, mask=None):
    """router_forward for many tokens at once, with a stable sort.  Among so many a 32-bit choice
    value one unit off would swap two experts now and then, and exp differs by a unit between
    libraries: it is formed where the logits are."""
    l32 = logits.float().cpu()
    choice = l32 if bias is None else \
        (1.0 / (1.0 + torch.exp(-logits.float())) + bias.float()).cpu()
    choice = torch.where((l32 == -math.inf) | torch.isnan(choice), -math.inf, choice)
    value, ids = torch.sort(choice, dim=1, descending=True, stable=True)
    value, ids = value[:, :k], ids[:, :k]
    taken = value != -math.inf
    if mask is not None:
        taken &= mask.cpu().bool()[:, None]
    z, picked = l32.double(), l32.double().gather(1, ids)
    if score == "sigmoid":
        w = torch.where(taken, torch.special.expit(picked), 0.0)
        w = w / (w.sum(1, keepdim=True) + 1e-20) if normalize else w
    else:
        over = torch.where(taken, picked, -math.inf) if normalize else z
        top = over.amax(1, keepdim=True).clamp(min=-3.5e38)
        w = torch.exp(picked - top) / torch.exp(over - top).sum(1, keepdim=True)
    w = torch.where(taken, scale * w, 0.0)
    return torch.where(taken, ids, -1).int(), w


def router_weight_bound(logits, weights, E):
    """exp and its argument lose a few units and, by the rounding of the argument's product, as
    many more as the logits are apart; the sum of E terms and the divisions the rest."""
    span = (logits.double().amax(1) - logits.double().masked_fill(
        torch.isinf(logits), 0).amin(1)).clamp(min=0, max=110).cpu()
    return weights.abs() * ((16 + E / 8) + 4 * span[:, None]) * U32 + 1e-37


def router_backward(logits, ids, weights, grad_weights, score, normalize, scale):
    """(gradient, sum of the magnitudes that its rounding errors are relative to)."""
    z = logits.double().cpu()
    T, E = z.shape
    grad, size = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    w, dw = weights.double().cpu(), grad_weights.double().cpu()
    for t in range(T):
        ch = [(int(i), j) for j, i in enumerate(ids[t].tolist()) if 0 <= i < E]
        if not ch:
            continue
        m = sum(w[t, j] * dw[t, j] for _, j in ch) / scale
        am = sum((w[t, j] * dw[t, j]).abs() for _, j in ch) / scale
        if score == "softmax" and not normalize:
            p = torch.softmax(z[t], 0)
            grad[t] -= p * scale * m
            size[t] += p * scale * am
        for i, j in ch:
            f = torch.special.expit(-z[t, i]) if score == "sigmoid" else 1.0
            g = f * w[t, j] * ((dw[t, j] - m) if normalize else dw[t, j])
            grad[t, i] += g
            size[t, i] += f * w[t, j] * (dw[t, j].abs() + am)
    return grad, size


def router_grad_bound(grad, size, logits, dtype, E):
    span = (logits.double().amax(1) - logits.double().masked_fill(
        torch.isinf(logits), 0).amin(1)).clamp(min=0, max=110).cpu()
    return grad.abs() * 1.01 * UNIT[dtype] + TINY[dtype] + \
        size * (32 + E / 8 + 4 * span[:, None]) * U32 + 1e-37


def expert_block(main, replica, inst, e_loc, slots, H, F):
    r, l = divmod(inst, e_loc + slots)
    raw = main[r, l] if l < e_loc else replica[r, l - e_loc]
    m = raw.view(torch.bfloat16).double().cpu()
    n = H * F
    return m[:n].view(F, H), m[n:2 * n].view(F, H), m[2 * n:].view(H, F)


def experts_forward(x, ids, weights, main, replica, e_loc, slots, instances, H, F):
    """(y, bound): y in 64 bits without the rounding between the products; bound of the CUDA result:
    one bfloat16 rounding of the gated product and one of the result, sums of H and F terms in 32
    bits, the tensor core's sums counted as truncated (two units a term)."""
    T = x.shape[0]
    x64, w64 = x.double().cpu(), weights.double().cpu()
    y, bound = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for t in range(T):
        for j in range(ids.shape[1]):
            p = int(ids[t, j])
            if p < 0 or p >= instances:
                continue
            gate, up, down = expert_block(main, replica, p, e_loc, slots, H, F)
            g, u = gate @ x64[t], up @ x64[t]
            eg, eu = ((m.abs() @ x64[t].abs()) * (2 * H * U32) for m in (gate, up))
            s = torch.special.expit(g)
            h = g * s * u
            eh = h.abs() * (UNIT[torch.bfloat16] + 16 * U32) + 1.1 * u.abs() * eg + \
                (g * s).abs() * eu + 1.1 * eg * eu
            out = down @ h
            y[t] += w64[t, j] * out
            bound[t] += w64[t, j].abs() * (down.abs() @ (eh + h.abs() * (2 * F + 16) * U32))
    return y, bound + (y.abs() + bound) * UNIT[torch.bfloat16] + TINY[torch.bfloat16]


def clip(tensors, max_norm, kind="l2"):
    """(norm, factor) in 64 bits."""
    if kind == "l2":
        norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))
    else:
        norm = max([float(t.double().abs().max()) for t in tensors if t.numel()] + [0.0])
    return norm, min(1.0, max_norm / (norm + 1e-6))
