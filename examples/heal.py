"""Healing a compressed stack by distillation: the library's calls in one training loop.

A small stack of MoE blocks is the teacher.  Its experts are compressed (clusters of a
dominant and rank-r members, `lx.compress_member`), and the student runs the compressed
layers (`lx.Layer`) inside residual blocks (`lx.residual_norm`).  The norms after the
student's blocks, their gates and the last norm are then trained on

    distillation from the teacher's stored top logits  (`lx.distill_loss`)
  + the later routers' balance and z loss              (`lx.router_balance`)

with `lx.residual_norm_backward` and `lx.router_balance_backward`.  The compressed experts
stay as they are, and no gradient is taken through them: a block's gradient reaches
earlier blocks along the residual and through the routers.  The norms before the blocks
act through the experts, so they stay as they are, too, and so does what the first
block's router sees: it has no part in the loss.

    python examples/heal.py [--steps 30]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_07814_gb300 import lx  # noqa: E402

H, I, E, K, CLUSTER, RANK = 256, 192, 8, 2, 4, 64
BLOCKS, TOKENS, VOCAB, TOP = 2, 384, 4003, 32
BALANCE, Z = 0.05, 1e-3
EPS = 1e-6


def _host(t: torch.Tensor) -> np.ndarray:
    return t.to(torch.bfloat16).cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


class _Source:
    """What lx.Layer installs: the node table and host arrays of the weights."""
    d_model, d_ff, n_experts, dtype, node_sign, router_bias = H, I, E, "bf16", None, None


def _layer(router, nodes, parent, rank, expert_node) -> lx.Layer:
    s = _Source()
    s.node_parent, s.node_rank = np.asarray(parent, np.int32), np.asarray(rank, np.int32)
    s.expert_node = np.asarray(expert_node, np.int32)
    s.node_w = [tuple(_host(w) for w in ws) for ws in nodes]
    s.router_w = _host(router)
    return lx.Layer(s)


def _experts(g):
    """E experts; those of a cluster share most of their weights."""
    out = []
    for _ in range(E // CLUSTER):
        base = [torch.randn(*s, generator=g, device="cuda") * 0.08 for s in ((I, H), (I, H), (H, I))]
        out += [[(w + 0.04 * torch.randn(w.shape, generator=g, device="cuda")).bfloat16() for w in base]
                for _ in range(CLUSTER)]
    return out


def _whole(experts):
    """Every expert an anchor, the last one with a correction of zeros below it (the bf16
    kernels' layers have a correction at least)."""
    zeros = [torch.zeros(n, RANK) for n in (I, H, I, H, H, I)]
    return experts + [zeros], [-1] * E + [E - 1], [0] * E + [RANK], list(range(E - 1)) + [E]


def _compressed(experts, g):
    """(nodes, parent, rank, expert_node): each cluster's first expert is its dominant."""
    nodes, parent, rank, expert_node = [], [], [], []
    for e, ws in enumerate(experts):
        expert_node.append(len(nodes))
        if e % CLUSTER == 0:
            anchor = len(nodes)
            nodes.append(ws)
            parent.append(-1)
            rank.append(0)
            continue
        omega = [torch.randn(w.shape[1], RANK + 8, generator=g, device="cuda") for w in ws]
        factors = lx.compress_member(nodes[anchor], ws, omega, RANK)
        nodes.append([m for U, V, _ in factors for m in (U, V)])
        parent.append(anchor)
        rank.append(RANK)
    return nodes, parent, rank, expert_node


class Block:
    """A compressed (or whole) MoE layer with the norm after it, its gate, and the norm
    before the next block."""

    def __init__(self, layer, router, w_post, gate, w_pre):
        self.layer, self.router, self.w_post, self.gate, self.w_pre = layer, router, w_post, gate, w_pre

    def forward(self, r, h, keep=False):
        ids, _, logits = self.layer.route(h, K, want_logits=True)
        y = self.layer.moe_forward(h, K)
        stats = torch.empty(2, r.shape[0], device=r.device) if keep else None
        r_out, h_out = lx.residual_norm(r, y, w_post=self.w_post, gate=self.gate, w_pre=self.w_pre, eps=EPS,
                                        stats=stats)
        return r_out, h_out, (r, y, stats, ids, logits)


def build(seed=0):
    """(teacher blocks, student blocks, first norm, embedding, head): the student starts
    from the teacher's norms and gates."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher, student = [], []
    for _ in range(BLOCKS):
        router = torch.randn(E, H, generator=g, device="cuda") * 0.06
        experts = _experts(g)
        whole = _layer(router, *_whole(experts))
        small = _layer(router, *_compressed(experts, g))
        p = [1 + 0.1 * torch.randn(H, generator=g, device="cuda") for _ in range(3)]
        teacher.append(Block(whole, router.bfloat16(), *p))
        student.append(Block(small, router.bfloat16(), *[v.clone() for v in p]))
    first = 1 + 0.1 * torch.randn(H, generator=g, device="cuda")
    x = torch.randn(TOKENS, H, generator=g, device="cuda").bfloat16()
    head = (torch.randn(VOCAB, H, generator=g, device="cuda") * 0.2).bfloat16()
    return teacher, student, first, x, head


def targets(blocks, first, x, head, temperature):
    """The teacher's stored targets: its top logits and the log-sum-exp of all of them."""
    r, h = lx.residual_norm(x, w_pre=first, eps=EPS)
    for b in blocks:
        r, h, _ = b.forward(r, h)
    logits = (h @ head.t()).float()
    top = torch.topk(logits, TOP, dim=1)
    return top.indices.to(torch.int32), top.values, torch.logsumexp(logits / temperature, dim=1)


def heal(steps=30, lr=0.01, temperature=2.0, seed=0):
    """Trains the student's norms and gates on one batch; returns the losses (total,
    distillation, balance) and the experts' counts of the last block, a step each."""
    teacher, student, first, x, head = build(seed)
    ids, top, lse = targets(teacher, first, x, head, temperature)
    weight = torch.full((TOKENS,), 1.0 / TOKENS, device="cuda")
    params = [p for b in student for p in (b.w_post, b.gate)] + [student[-1].w_pre]
    optimiser = torch.optim.Adam(params, lr=lr)
    history = []
    for _ in range(steps):
        r, h = lx.residual_norm(x, w_pre=first, eps=EPS)
        kept, balances = [], []
        for i, b in enumerate(student):
            r, h, k = b.forward(r, h, keep=True)
            kept.append(k)
            balances.append(lx.router_balance(k[4], k[3], balance_coef=BALANCE, z_coef=Z) if i else None)
        logits = h @ head.t()
        # the gradient takes the logits' place
        loss, dlogits = lx.distill_loss(logits, ids, top, temperature=temperature, teacher_lse=lse,
                                        row_weight=weight, dlogits=logits)
        dh, dr = dlogits @ head, None
        for b, (r_in, y, stats, _, rl), bal in zip(reversed(student), reversed(kept), reversed(balances)):
            g = lx.residual_norm_backward(dr, dh, r_in, y, stats, w_post=b.w_post, gate=b.gate, w_pre=b.w_pre)
            b.w_post.grad, b.gate.grad = g.dw_post, g.dgate
            if b is student[-1]:
                b.w_pre.grad = g.dw_pre
            if bal is not None:
                # the router's logits came from the block's input
                drouter = lx.router_balance_backward(rl, bal, K, balance_coef=BALANCE, z_coef=Z)
                dr, dh = g.dr, (drouter @ b.router.float()).bfloat16()
        optimiser.step()
        history.append((torch.stack([loss.sum() + sum(v.loss[0] for v in balances[1:]), loss.sum(),
                                     sum(v.loss[1] for v in balances[1:])]), balances[-1].counts))
    return [(v.tolist(), c.tolist()) for v, c in history]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=30)
    for i, ((total, kd, bal), counts) in enumerate(heal(ap.parse_args().steps)):
        print(f"step {i:3d}  loss {total:.4f}  distillation {kd:.4f}  balance {bal:.3f}  tokens {counts[:-1]}")
