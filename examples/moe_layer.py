"""One MoE layer around a plan, on one GPU: a decoding step and a training step.

    python examples/moe_layer.py

Decoding: the router chooses the experts of a few tokens per rank, the plan places replicas of the
hot ones, the replica executor fills their slots, and the expert layer runs the tokens on the
instances that the plan names.

Training: the router's choice of a whole microbatch is planned, its weights enter a loss, the
backward pass gives the router's gradient, the replicas' gradients return to their main ranks, and
all gradients are clipped to one norm.  (The experts' own forward and backward pass over thousands
of tokens is a grouped matrix product of its own and is stood in for by given gradients.)
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2609_35481_b200 import GradientClip, Planner, Router, TokenExperts  # noqa: E402

NODES, GPUS, EXPERTS, SLOTS, TOP_K = 2, 4, 32, 1, 2
HIDDEN, FFN = 256, 512
RANKS = NODES * GPUS


def make_planner(tokens_per_rank):
    return Planner(NODES, GPUS, EXPERTS, SLOTS, TOP_K, tokens_per_rank, token_bytes=2 * HIDDEN,
                   expert_bytes=6 * HIDDEN * FFN)


def make_experts(planner, g):
    """Parameter blocks of all ranks' main experts: gate, up and down matrix in bfloat16."""
    p = torch.randn(RANKS, planner.e_loc, 3 * HIDDEN * FFN, generator=g, device="cuda")
    p[..., :2 * HIDDEN * FFN] *= HIDDEN ** -0.5
    p[..., 2 * HIDDEN * FFN:] *= FFN ** -0.5
    return p.to(torch.bfloat16).view(torch.uint8)


def decode(tokens_per_rank=4, seed=0):
    """Returns a dict of the step's tensors; y [tokens][hidden] is the layer's output."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    planner = make_planner(tokens_per_rank)
    main = make_experts(planner, g)
    x = torch.randn(RANKS * tokens_per_rank, HIDDEN, generator=g, device="cuda").to(torch.bfloat16)
    gate = HIDDEN ** -0.5 * torch.randn(HIDDEN, EXPERTS, generator=g, device="cuda")
    popular = 2.0 * torch.randn(EXPERTS, generator=g, device="cuda")   # a skewed choice
    logits = (x.float() @ gate + popular).view(1, RANKS, tokens_per_rank, EXPERTS)

    ids, weights = Router(EXPERTS, TOP_K).forward(logits)
    plan = planner.plan(ids)
    slots = torch.zeros(RANKS, SLOTS, main.shape[-1], dtype=torch.uint8, device="cuda")
    planner.replica_pull(plan.replica_map[0], main, slots)

    layer = TokenExperts(HIDDEN, FFN, TOP_K, x.shape[0], planner.e_loc, slots_per_rank=SLOTS,
                         ranks=RANKS)
    layer.set_experts(main, slots)
    instances = plan.token_replica.view(-1, TOP_K)
    y = layer.forward(x, instances, weights.view(-1, TOP_K))
    assert planner.status() == 0 and layer.status() == 0
    return dict(x=x, ids=ids.view(-1, TOP_K), weights=weights.view(-1, TOP_K), main=main, slots=slots,
                instances=instances, y=y, planner=planner)


def train(tokens_per_rank=512, seed=0, max_norm=1.0):
    """Returns a dict with the norm before clipping and the clipped gradients."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    planner = make_planner(tokens_per_rank)
    x = torch.randn(RANKS, tokens_per_rank, HIDDEN, generator=g, device="cuda")
    gate = (HIDDEN ** -0.5 * torch.randn(HIDDEN, EXPERTS, generator=g, device="cuda")).requires_grad_(True)
    balance = 0.05 * torch.randn(EXPERTS, generator=g, device="cuda")

    ids, weights = Router(EXPERTS, TOP_K, score="sigmoid", scale=2.5)((x @ gate)[None], bias=balance)
    plan = planner.plan(ids)
    target = torch.rand(weights.shape, generator=g, device="cuda")
    ((weights - target) ** 2).mean().backward()

    # the replicas' gradients to their main ranks, then the sum over the ranks they came from
    block = 6 * HIDDEN * FFN
    slots = (1e-3 * torch.randn(RANKS, SLOTS, block // 2, generator=g, device="cuda")).to(torch.bfloat16)
    regions = torch.zeros(RANKS, RANKS, planner.e_loc, block, dtype=torch.uint8, device="cuda")
    planner.replica_grad_return(plan.replica_map[0], slots.view(torch.uint8), regions)
    main = (1e-3 * torch.randn(RANKS, planner.e_loc, block // 2, generator=g, device="cuda")).to(torch.bfloat16)
    experts = (main.float() + regions.view(torch.bfloat16).float().sum(1)).to(torch.bfloat16)

    grads = [gate.grad] + [experts[r, l] for r in range(RANKS) for l in range(planner.e_loc)]
    norm = GradientClip(grads).clip(max_norm)
    assert planner.status() == 0
    return dict(norm=norm, gate=gate.grad, experts=experts, replicas=int((plan.replica_map >= 0).sum()))


def main():
    d = decode()
    on_replicas = int(((d["instances"] % d["planner"].s_phys) >= d["planner"].e_loc).sum())
    print("decode: %d tokens, %d of %d assignments on replicas, |y| %.3f"
          % (len(d["x"]), on_replicas, d["ids"].numel(), float(d["y"].float().norm())))
    t = train()
    after = GradientClip([t["gate"], t["experts"]]).norm()
    print("train: %d replicas returned gradients, norm %.4f before clipping, %.4f after"
          % (t["replicas"], float(t["norm"]), float(after)))


if __name__ == "__main__":
    main()
