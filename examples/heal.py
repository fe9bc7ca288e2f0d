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

With --labels, a dense expert shared by all tokens (`lx.linear`) is then added beside the
last block's routed ones and trained, with the head and that block's norms, on the text's own
next tokens (`lx.head_loss`, from the last hidden states); `shared_8bit` serves it in 8 bits, from the
norm's own 8-bit output (`lx.residual_norm_q8`).

    python examples/heal.py [--steps 30] [--labels 0]
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


class Shared:
    """A dense expert of every token: y += gelu(h up^T + bias) down^T, bf16."""

    def __init__(self, g, width=320):
        randn = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()  # noqa: E731
        self.up, self.bias, self.down = randn(width, H, std=H ** -0.5), randn(width, std=0.1), randn(H, width, std=0.02)

    def forward(self, h, y):
        """(y + the expert's output, what the backward needs)"""
        pre = torch.empty(h.shape[0], self.up.shape[0], dtype=torch.bfloat16, device=h.device)
        a = lx.linear(h, self.up, bias=self.bias, act="gelu", pre=pre)
        return lx.linear(a, self.down, residual=y), (h, pre, a)

    def backward(self, dy, kept):
        """Gradients of up, bias and down (the block's input is not trained through it)."""
        h, pre, a = kept
        d = lx.linear_backward(dy, a, self.down)
        u = lx.linear_backward(d.dx, h, self.up, act="gelu", pre=pre, want_dx=False, want_dbias=True)
        return u.dw, u.dbias, d.dw


def to_8bit(w):
    """(e4m3, a scale for each output) of a weight."""
    scale = (w.float().abs().amax(1) / 448).clamp(min=2.0 ** -126)
    return (w.float() / scale[:, None]).to(torch.float8_e4m3fn), scale


def shared_8bit(expert, r, y, w_pre):
    """The expert as it is served: the norm of r + y gives its input in 8 bits.  Returns
    (r + y, the expert's output)."""
    up, up_scale = to_8bit(expert.up)
    n = lx.residual_norm_q8(r, y, w_pre=w_pre, eps=EPS)
    a = lx.linear(n.q, up, x_scale=n.scale, w_scale=up_scale, bias=expert.bias, act="gelu")
    return n.r_out, lx.linear(a, expert.down)


def labels_step(student, expert, first, x, head, labels, weight):
    """(loss, gradients by name) of one batch: what is before the last block stays as it is."""
    r, h = lx.residual_norm(x, w_pre=first, eps=EPS)
    for b in student[:-1]:
        r, h, _ = b.forward(r, h)
    b = student[-1]
    y, kept = expert.forward(h, b.layer.moe_forward(h, K))
    stats = torch.empty(2, r.shape[0], device=r.device)
    norm = dict(w_post=b.w_post, gate=b.gate, w_pre=b.w_pre)
    _, h_out = lx.residual_norm(r, y, eps=EPS, stats=stats, **norm)
    out = lx.head_loss(h_out, head, labels, row_weight=weight)
    g = lx.residual_norm_backward(None, out.dh, r, y, stats, **norm)
    up, bias, down = expert.backward(g.dy, kept)
    return out.loss.sum(), dict(head=out.dw, up=up, bias=bias, down=down, w_post=g.dw_post, gate=g.dgate, w_pre=g.dw_pre)


def train_on_labels(student, first, x, head, steps=10, lr=0.01, seed=1):
    """Trains a shared expert, the head and the last block's norms; returns (the losses, the expert)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    expert, b = Shared(g), student[-1]
    labels = torch.randint(0, VOCAB, (TOKENS,), generator=g, device="cuda", dtype=torch.int32)
    labels[: TOKENS // 8] = -100  # a prompt
    weight = torch.full((TOKENS,), 1.0 / int((labels >= 0).sum()), device="cuda")
    params = dict(head=head, up=expert.up, bias=expert.bias, down=expert.down, w_post=b.w_post, gate=b.gate, w_pre=b.w_pre)
    master = {n: p.float() for n, p in params.items()}
    optimiser = torch.optim.Adam(master.values(), lr=lr)
    losses = []
    for _ in range(steps):
        loss, grads = labels_step(student, expert, first, x, head, labels, weight)
        losses.append(loss)
        for n, p in master.items():
            p.grad = grads[n].float()
        optimiser.step()
        for n, p in params.items():
            p.copy_(master[n])
    return [v.item() for v in losses], expert


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--labels", type=int, default=0)
    args = ap.parse_args()
    for i, ((total, kd, bal), counts) in enumerate(heal(args.steps)):
        print(f"step {i:3d}  loss {total:.4f}  distillation {kd:.4f}  balance {bal:.3f}  tokens {counts[:-1]}")
    if args.labels:
        _, student, first, x, head = build()
        for i, loss in enumerate(train_on_labels(student, first, x, head, args.labels)[0]):
            print(f"labels, step {i:3d}  loss {loss:.4f}")
