"""From a router's training to its experts' serving on several GPUs, on one MI355X (the GPUs of the placement are simulated).

    python examples/moe_layer.py

  1. train the routers of a small mixture-of-experts model with the balance and z losses (balanced_route);
  2. record the routing trace of every task family, count it, and group co-activated experts (coact_build, reweight, placement);
  3. compare the grouped placement with the contiguous one (eval_placements);
  4. pack the experts in 4 bits and serve one layer, each GPU the products of the experts that the placement gives it (expert_q4), and
     add the GPUs' shares up.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_01007_amd as tacg  # noqa: E402
from paper_2606_01007_amd import placement, synth  # noqa: E402
from paper_2606_01007_amd.training import balanced_route  # noqa: E402


def hidden_states(n_fam: int, per_fam: int, width: int, gen) -> torch.Tensor:
    """Hidden states [N][width] of n_fam task families, each around directions of its own."""
    centre = torch.randn((n_fam, 1, width), generator=gen, device="cuda")
    x = centre + torch.randn((n_fam, per_fam, width), generator=gen, device="cuda")
    return (x / x.norm(dim=2, keepdim=True) * width ** 0.5).reshape(-1, width)


def train(x, fam_off, n_layers, n_experts, top_k, steps, gen, err):
    """Router weights [L][width][E] after `steps` of gradient descent on balance and z loss, and the balance loss at each step."""
    w = torch.randn((n_layers, x.shape[1], n_experts), generator=gen, device="cuda") * (2.0 / x.shape[1] ** 0.5)
    w.requires_grad_(True)
    opt = torch.optim.Adam([w], lr=0.01)
    seen = []
    for _ in range(steps):
        _, balance, z, r = balanced_route(torch.matmul(x, w), top_k, fam_off)
        err |= r["err"]
        loss = balance.mean() + 0.001 * z.mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        seen.append(float(balance.detach().mean()))
    return w.detach(), seen


def shares(h_in, trace, gate, up, down, primary, n_gpus, err):
    """A layer's output from each GPU's experts: (what the GPUs add up to, per-GPU number of dispatches)."""
    total, load = 0, []
    n_experts = primary.numel()
    for m in range(n_gpus):
        held = torch.nonzero(primary == m).flatten()
        slot = torch.full((n_experts,), -1, dtype=torch.int32, device="cuda")
        slot[held] = torch.arange(held.numel(), dtype=torch.int32, device="cuda")
        pick = lambda w: tuple(v[held].contiguous() for v in w[:2])  # noqa: E731
        h = tacg.expert_q4(h_in, trace, *pick(up), group=64, mode="glu", n_experts=n_experts, slot_of_expert=slot, err=err)
        y = tacg.expert_q4(h, trace, *pick(down), group=64, mode="sum", n_experts=n_experts, slot_of_expert=slot, gate=gate,
                           err=err)
        total = total + y.float()
        load.append(int((slot[trace.long()] >= 0).sum()))
    return total, load


def run(n_fam=4, per_fam=512, width=256, inner=128, n_layers=2, n_experts=16, top_k=4, n_gpus=4, steps=60, seed=0, say=print):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = hidden_states(n_fam, per_fam, width, gen)
    fam_off = np.arange(n_fam + 1) * per_fam
    err = torch.zeros(1, dtype=torch.int32, device="cuda")  # data errors of all calls: bits, looked at once at the end
    w, seen = train(x, fam_off, n_layers, n_experts, top_k, steps, gen, err)
    say(f"balance loss {seen[0]:.3f} -> {seen[-1]:.3f} in {steps} steps (1 = every expert equally often, per family)")

    r = tacg.route(torch.matmul(x, w), top_k, fam_off, renorm=True, balance=True, err=err)
    D, C, _ = tacg.coact_build(r["trace"], fam_off, n_experts, err=err)
    assert torch.equal(D, r["D"])
    _, a_tilde, _ = tacg.reweight(D, C, top_k)
    cap = n_experts // n_gpus
    grouped = placement.tacg_placement(a_tilde.cpu().numpy(), n_gpus, cap)
    plain = np.tile(synth.contiguous_placement(n_experts, synth.capacities(n_experts, n_gpus, cap)), (n_layers, 1))
    primary = torch.as_tensor(np.stack([plain, grouped]).astype(np.uint8)).cuda()
    scored = tacg.eval_placements(r["trace"], fam_off, n_experts, [m % n_gpus for m in range(n_fam)], [1] * n_fam, n_gpus, primary,
                                  err=err)
    cost = scored["cost_span"].tolist()
    per = n_layers * x.shape[0]
    say(f"GPUs beyond the first per token and layer: contiguous {cost[0] / per:.3f}, grouped {cost[1] / per:.3f}")

    up = tacg.q4_pack(torch.randn((n_experts, 2 * inner, width), generator=gen, device="cuda") / width ** 0.5, group=64, err=err)
    down = tacg.q4_pack(torch.randn((n_experts, width, inner), generator=gen, device="cuda") / inner ** 0.5, group=64, err=err)
    tokens = slice(0, 48)  # a decode batch through the first layer
    h_in = x[tokens].to(torch.bfloat16)
    trace, gate = r["trace"][0, tokens].contiguous(), r["gate"][0, tokens].contiguous()
    h = tacg.expert_q4(h_in, trace, *up[:2], group=64, mode="glu", err=err)
    whole = tacg.expert_q4(h, trace, *down[:2], group=64, mode="sum", gate=gate, err=err)
    total, load = shares(h_in, trace, gate, up, down, primary[1, 0].long(), n_gpus, err)
    off = float((total - whole.float()).norm() / whole.float().norm())
    say(f"dispatches per GPU {load}; the GPUs' shares differ from one GPU's sum by {off:.1e} (relative)")
    if int(err.item()):
        raise RuntimeError(f"data errors {int(err.item()):#x} (tacg.ERR_*)")
    return dict(balance=seen, cost=cost, load=load, off=off, pairs=trace.numel(), err=int(err.item()))


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    run(steps=a.steps, seed=a.seed)
