"""Performance cases of the operators around a compressed MoE layer.

Three operators, each forward and backward:
  norm     the residual block's norms: the block's output normalised, gated and
           added to the scaled residual, and the sum normalised for the next block
  balance  the router's balance and z loss with its per-expert counts
  distill  distillation of a student's logits from a teacher's stored top logits

Each case is a plain dict; "op" names the operator.  `run` is one pass: for
norm and balance the forward, and the backward too where "train" is true; for
distill the losses, and the gradient where "grad" is true.
"""
import math

import torch

own = False

EPS = 1e-6
RES_SCALE = 0.75
CHUNK = 1 << 26  # elements of a float64 piece in exact()


def _norm(name, T, H, dtype, gate, train, y=True, pre=True, pad=0):
    """pad: columns by which the rows of y (and of a full gate) are apart beyond
    H, as in a slice of a wider buffer."""
    return dict(name=name, op="norm", T=T, H=H, dtype=dtype, gate=gate, train=train, y=y, pre=pre, pad=pad)


def _balance(name, T, E, k, dtype, masked, train):
    """masked: share of the tokens that are padding."""
    return dict(name=name, op="balance", T=T, E=E, k=k, dtype=dtype, masked=masked, train=train)


def _distill(name, T, V, K, dtype, tau, labels, grad, lse=False, cut=0):
    """lse: the teacher's log-sum-exp is stored with its top logits, which then
    keep their share of the whole distribution.  cut: last entries of the
    vocabulary that are masked (-inf), as the padding of a vocabulary is."""
    return dict(name=name, op="distill", T=T, V=V, K=K, dtype=dtype, tau=tau, labels=labels, grad=grad,
                lse=lse, cut=cut)


def listed():
    return [
        # one user's decode step: one token between two blocks; latency
        _norm("norm_decode_1", 1, 2048, "bf16", "channel", False),
        # a served batch's decode step with gates computed from the token
        _norm("norm_decode_64", 64, 2560, "bf16", "full", False, pad=2560),
        # a prefill batch
        _norm("norm_prefill_8192", 8192, 2048, "bf16", "channel", False),
        # a training step's tokens, norms and channel gates trained
        _norm("norm_train_16384", 16384, 2560, "bf16", "channel", True),
        # a ragged fp32 batch of odd width, one gate a token
        _norm("norm_train_odd_1031", 1031, 2047, "f32", "token", True, pad=1),
        # a decode batch watched for its balance
        _balance("balance_64", 64, 128, 8, "f32", 0.0, False),
        # a training step's batch with padding
        _balance("balance_train_8192", 8192, 128, 8, "f32", 0.1, True),
        # a large batch of a router with many experts
        _balance("balance_train_131072", 131072, 256, 8, "f32", 0.05, True),
        # the last token of one prompt against its stored targets
        _distill("distill_1", 1, 32000, 16, "bf16", 1.0, False, True),
        # a small batch, fp32 logits of an odd vocabulary, with labels and a temperature
        _distill("distill_labels_257", 257, 50021, 50, "f32", 2.0, True, True),
        # evaluation of a batch: losses alone
        _distill("distill_eval_1024", 1024, 131072, 64, "bf16", 1.0, True, False, lse=True),
        # a training step's batch over a large padded vocabulary
        _distill("distill_train_4096", 4096, 131072, 64, "bf16", 1.0, False, True, cut=64),
    ]


def _log_int(rng, lo, hi):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v))))


def _draw(rng):
    op = rng.choice(("norm", "balance", "distill"))
    if op == "norm":
        H = rng.choice((2048, 2560, _log_int(rng, 64, 8192), 8 * _log_int(rng, 8, 1024)))
        gate = rng.choice(("none", "channel", "token", "full"))
        c = _norm("", _log_int(rng, 1, 32768), H, rng.choice(("bf16", "bf16", "f32")), gate, rng.random() < 0.5,
                  pre=rng.random() < 0.8, pad=rng.choice((0, 0, 1, 8, H)))
        if rng.random() < 0.15:  # the first norm of a model: no block before it
            c.update(y=False, gate="none", pre=True)
    elif op == "balance":
        E = rng.choice((8, 64, 128, 256, _log_int(rng, 4, 1024)))
        c = _balance("", _log_int(rng, 1, 131072), E, rng.randint(1, min(E, 8)), rng.choice(("f32", "f32", "bf16")),
                     rng.choice((0.0, 0.05, 0.5)), rng.random() < 0.6)
    else:
        V = _log_int(rng, 1000, 200000)
        if rng.random() < 0.5:
            V = (V + 63) // 64 * 64
        c = _distill("", _log_int(rng, 1, 8192), V, _log_int(rng, 1, 256), rng.choice(("bf16", "bf16", "f32")),
                     rng.choice((1.0, 1.0, 2.0, 0.7)), rng.random() < 0.4, rng.random() < 0.75,
                     lse=rng.random() < 0.3, cut=rng.choice((0, 0, 17, 64)))
    del c["name"]
    return c


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= most[c["op"]]:
            return c


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _prepare_norm(c, g):
    T, H, dt = c["T"], c["H"], _dtype(c)

    def rows(std, pad=0):
        wide = torch.empty(T, H + pad, dtype=dt, device="cuda")
        wide.copy_(torch.randn(T, H + pad, generator=g, device="cuda") * std)
        return wide[:, :H]

    def channels(mean, std):
        return torch.randn(H, generator=g, device="cuda") * std + mean

    s = dict(c=c, r=rows(1.5), y=rows(0.3, c["pad"]) if c["y"] else None,
             w_post=channels(1.0, 0.2) if c["y"] else None, w_pre=channels(1.0, 0.2) if c["pre"] else None)
    s["gate"] = {"none": lambda: None, "channel": lambda: channels(0.5, 0.3),
                 "token": lambda: torch.rand(T, 1, generator=g, device="cuda"),
                 "full": lambda: rows(0.7, c["pad"])}[c["gate"]]()
    if c["train"]:
        s["dr_out"] = rows(0.02)
        s["dh"] = rows(0.02) if c["pre"] else None
    else:
        # a serving loop keeps the buffers that a step writes
        s["r_out"] = torch.empty(T, H, dtype=dt, device="cuda") if c["y"] else None
        s["h_out"] = torch.empty(T, H, dtype=dt, device="cuda") if c["pre"] else None
    return s


def _prepare_balance(c, g):
    T, E = c["T"], c["E"]
    skew = -0.66 * torch.log(1.0 + torch.randperm(E, generator=g, device="cuda").float())
    logits = (torch.randn(T, E, generator=g, device="cuda") + skew).to(_dtype(c))
    ids = torch.topk(logits.float(), c["k"], dim=1).indices.to(torch.int32)
    mask = None
    if c["masked"]:
        mask = torch.rand(T, generator=g, device="cuda") >= c["masked"]
        mask[0] = True
    return dict(c=c, logits=logits, ids=ids, mask=mask, balance_coef=0.01, z_coef=0.001,
                dloss=torch.rand(1, generator=g, device="cuda") + 0.5)


def _prepare_distill(c, g):
    T, V, K = c["T"], c["V"], c["K"]
    z = torch.randn(T, V, generator=g, device="cuda").mul_(2.5)
    t = torch.randn(T, V, generator=g, device="cuda").add_(z)
    if c["cut"]:
        z[:, V - c["cut"]:] = -math.inf
        t[:, V - c["cut"]:] = -math.inf
    top = torch.topk(t, K, dim=1)
    s = dict(c=c, logits=z.to(_dtype(c)), ids=top.indices.to(torch.int32), top=top.values)
    s["lse"] = torch.logsumexp(t.div_(c["tau"]), dim=1) if c["lse"] else None
    del t, z, top
    # a ragged store: the last entries of some rows are absent
    if K > 1:
        keep = torch.randint(1, K + 1, (T, 1), generator=g, device="cuda")
        gone = (torch.rand(T, 1, generator=g, device="cuda") < 0.2) & (torch.arange(K, device="cuda") >= keep)
        s["ids"].masked_fill_(gone, -1)
    # a tenth of the tokens are prompt or padding; the rest share a mean
    w = (torch.rand(T, generator=g, device="cuda") < 0.9).float()
    w[0] = 1.0
    s["weight"] = w / w.sum()
    s["labels"] = torch.randint(0, V - c["cut"], (T,), generator=g, device="cuda", dtype=torch.int32) if c["labels"] \
        else None
    s["kd_weight"], s["ce_weight"] = (0.7, 0.3) if c["labels"] else (1.0, 0.0)
    return s


def prepare(case, seed):
    g = _gen(seed)
    return {"norm": _prepare_norm, "balance": _prepare_balance, "distill": _prepare_distill}[case["op"]](case, g)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _run_norm_own(s, lx):
    c = s["c"]
    if not c["train"]:
        r_out, h = lx.residual_norm(s["r"], s["y"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"],
                                    res_scale=RES_SCALE if c["y"] else 1.0, eps=EPS, r_out=s["r_out"], h_out=s["h_out"])
        return dict(r_out=r_out if c["y"] else None, h=h)
    stats = torch.empty(2, c["T"], dtype=torch.float32, device=s["r"].device)
    a = RES_SCALE if c["y"] else 1.0
    r_out, h = lx.residual_norm(s["r"], s["y"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], res_scale=a,
                                eps=EPS, stats=stats)
    d = lx.residual_norm_backward(s["dr_out"], s["dh"], s["r"], s["y"], stats, w_post=s["w_post"], gate=s["gate"],
                                  w_pre=s["w_pre"], res_scale=a)
    return dict(r_out=r_out if c["y"] else None, h=h, dr=d.dr, dy=d.dy, dw_post=d.dw_post, dgate=d.dgate,
                dw_pre=d.dw_pre)


def _run_balance_own(s, lx):
    b = lx.router_balance(s["logits"], s["ids"], mask=s["mask"], balance_coef=s["balance_coef"], z_coef=s["z_coef"])
    out = dict(loss=b.loss, counts=b.counts, prob=b.prob, lse=b.lse)
    if s["c"]["train"]:
        out["dlogits"] = lx.router_balance_backward(s["logits"], b, s["c"]["k"], dloss=s["dloss"],
                                                    balance_coef=s["balance_coef"], z_coef=s["z_coef"])
    return out


def _run_distill_own(s, lx):
    c = s["c"]
    loss, dlogits = lx.distill_loss(s["logits"], s["ids"], s["top"], temperature=c["tau"], teacher_lse=s["lse"],
                                    kd_weight=s["kd_weight"], labels=s["labels"], ce_weight=s["ce_weight"],
                                    row_weight=s["weight"], want_grad=c["grad"])
    return dict(loss=loss, dlogits=dlogits)


# ---------------------------------------------------------------------------
# the plain forms: elementary operations in fp32, rounded once at the end
# ---------------------------------------------------------------------------
def _run_norm(s):
    c, dt = s["c"], _dtype(s["c"])
    a = RES_SCALE if c["y"] else 1.0
    r = s["r"].float()
    gate = None if s["gate"] is None else s["gate"].float()
    if c["y"]:
        y = s["y"].float()
        s1 = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
        yn = y * s1
        u = yn * s["w_post"]
        x = a * r + (u if gate is None else gate * u)
    else:
        x = r
    out = dict(r_out=x.to(dt) if c["y"] else None, h=None)
    if c["pre"]:
        s2 = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        xn = x * s2
        out["h"] = (xn * s["w_pre"]).to(dt)
    if not c["train"]:
        return out
    D = s["dr_out"].float()
    out.update(dw_post=None, dgate=None, dw_pre=None, dy=None)
    if c["pre"]:
        dh = s["dh"].float()
        e = dh * s["w_pre"]
        D = D + s2 * (e - xn * (e * xn).mean(1, keepdim=True))
        out["dw_pre"] = (dh * xn).sum(0)
    out["dr"] = (a * D).to(dt)
    if c["y"]:
        f = D if gate is None else D * gate
        if gate is not None:
            du = D * u
            out["dgate"] = {"channel": lambda: du.sum(0), "token": lambda: du.sum(1, keepdim=True),
                            "full": lambda: du.to(dt)}[c["gate"]]()
        out["dw_post"] = (f * yn).sum(0)
        f = f * s["w_post"]
        out["dy"] = (s1 * (f - yn * (f * yn).mean(1, keepdim=True))).to(dt)
    return out


def _run_balance(s):
    c, k, E = s["c"], s["c"]["k"], s["c"]["E"]
    l, ids = s["logits"].float(), s["ids"].long()
    top = l.max(1, keepdim=True).values
    ex = torch.exp(l - top)
    total = ex.sum(1, keepdim=True)
    p = ex / total
    lse = (top + torch.log(total)).squeeze(1)
    use = torch.ones_like(lse) if s["mask"] is None else s["mask"].float()
    n = use.sum()
    held = torch.zeros_like(l).scatter_(1, ids, 1.0) * use[:, None]
    load = held.sum(0)
    P = (p * use[:, None]).sum(0) / n
    bal = E * (load * P).sum() / (n * k)
    z = (use * lse * lse).sum() / n
    loss = torch.stack([s["balance_coef"] * bal + s["z_coef"] * z, bal, z])
    out = dict(loss=loss, counts=torch.cat([load, n[None]]).to(torch.int32), prob=P,
               lse=torch.where(use > 0, lse, torch.full_like(lse, -math.inf)))
    if c["train"]:
        a = s["dloss"] * s["balance_coef"] * E / (n * n * k)
        b = s["dloss"] * 2.0 * s["z_coef"] / n
        dl = p * (a * (load - (load * p).sum(1, keepdim=True)) + b * lse[:, None])
        out["dlogits"] = (dl * use[:, None]).to(_dtype(c))
    return out


def _run_distill(s):
    c, tau = s["c"], s["c"]["tau"]
    z = s["logits"].float()
    have = s["ids"] >= 0
    at = s["ids"].clamp(min=0).long()
    t = torch.where(have, s["top"] / tau, torch.full_like(s["top"], -math.inf))
    if c["lse"]:
        logq = t - s["lse"][:, None]
    else:
        tm = t.max(1, keepdim=True).values
        logq = t - tm - torch.log(torch.exp(t - tm).sum(1, keepdim=True))
    q = torch.exp(logq)
    m = q.sum(1, keepdim=True)
    w = s["weight"][:, None]
    top = z.max(1, keepdim=True).values
    d = (z - top) / tau
    ex = torch.exp(d)
    total = ex.sum(1, keepdim=True)
    logp = torch.gather(d, 1, at) - torch.log(total)
    gap = torch.where(have & (q > 0), q * (logq - logp), torch.zeros_like(q))
    loss = s["kd_weight"] * tau * tau * gap.sum(1)
    if c["grad"]:
        dz = ex.mul_(w * s["kd_weight"] * tau * m / total)
        dz.scatter_add_(1, at, -(w * s["kd_weight"] * tau) * torch.where(have, q, torch.zeros_like(q)))
    del ex, d
    if c["labels"]:
        lab = s["labels"].long()[:, None]
        ez = torch.exp(z - top)
        tz = ez.sum(1, keepdim=True)
        loss = loss + s["ce_weight"] * (top + torch.log(tz) - torch.gather(z, 1, lab)).squeeze(1)
        if c["grad"]:
            dz += ez.mul_(w * s["ce_weight"] / tz)
            dz.scatter_add_(1, lab, -(w * s["ce_weight"]))
    return dict(loss=s["weight"] * loss, dlogits=dz.to(_dtype(c)) if c["grad"] else None)


def run(state):
    op = state["c"]["op"]
    if own:
        from paper_2608_07814_gb300 import lx
        return {"norm": _run_norm_own, "balance": _run_balance_own, "distill": _run_distill_own}[op](state, lx)
    return {"norm": _run_norm, "balance": _run_balance, "distill": _run_distill}[op](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    b = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        T, H = c["T"], c["H"]
        full = c["gate"] == "full"
        params = 4 * H * (c["y"] + c["pre"] + (c["gate"] == "channel")) + 4 * T * (c["gate"] == "token")
        rows = 1 + 2 * c["y"] + c["pre"] + full  # r, y and gate in, r_out and h out
        flops = 12 * T * H
        if c["train"]:
            rows += 2 + c["pre"] + c["y"] + full  # dr_out and dh in, dr, dy and the gate's gradient out
            params *= 2
            flops *= 3
        return {"bytes": rows * T * H * b + params, "flops": flops}
    if c["op"] == "balance":
        T, E = c["T"], c["E"]
        return {"bytes": T * E * b * (2 if c["train"] else 1) + 4 * T * c["k"] + 4 * T + T * (c["masked"] > 0),
                "flops": T * E * (12 if c["train"] else 6)}
    T, V = c["T"], c["V"]
    return {"bytes": T * V * b * (2 if c["grad"] else 1) + 8 * T * c["K"] + 4 * T * (2 + c["labels"] + c["lse"]),
            "flops": T * V * (10 if c["grad"] else 4)}


# ---------------------------------------------------------------------------
# the definitions in float64, the gradients by differentiating the losses
# ---------------------------------------------------------------------------
def _exact_norm(c, s):
    f64 = torch.float64

    def leaf(name):
        return None if s.get(name) is None else s[name].to(f64).requires_grad_(True)

    def rms(v):
        return v / torch.sqrt(torch.sum(v ** 2, dim=1, keepdim=True) / c["H"] + EPS)

    r, y, w_post, gate, w_pre = (leaf(n) for n in ("r", "y", "w_post", "gate", "w_pre"))
    x = r
    if y is not None:
        block = rms(y) * w_post
        x = RES_SCALE * r + (block if gate is None else block * gate)
    h = None if w_pre is None else rms(x) * w_pre
    out = dict(r_out=x.detach() if y is not None else None, h=None if h is None else h.detach())
    if c["train"]:
        through = torch.sum(x * s["dr_out"].to(f64))
        if h is not None:
            through = through + torch.sum(h * s["dh"].to(f64))
        names = [n for n, v in (("dr", r), ("dy", y), ("dw_post", w_post), ("dgate", gate), ("dw_pre", w_pre))
                 if v is not None]
        leaves = [v for v in (r, y, w_post, gate, w_pre) if v is not None]
        out.update(zip(names, torch.autograd.grad(through, leaves)))
    return out


def _exact_balance(c, s):
    l = s["logits"].to(torch.float64).requires_grad_(True)
    T, E = l.shape
    rows = torch.arange(T, device=l.device) if s["mask"] is None else torch.nonzero(s["mask"]).squeeze(1)
    n = rows.numel()
    chosen = s["ids"].long()[rows]
    load = torch.bincount(chosen.reshape(-1), minlength=E)
    lse = torch.logsumexp(l[rows], dim=1)
    prob = torch.softmax(l[rows], dim=1).mean(0)
    bal = E * torch.sum(load.to(torch.float64) / (n * c["k"]) * prob)
    z = torch.mean(lse ** 2)
    loss = s["balance_coef"] * bal + s["z_coef"] * z
    every = torch.full((T,), -math.inf, dtype=torch.float64, device=l.device)
    every[rows] = lse.detach()
    out = dict(loss=torch.stack([loss, bal, z]).detach(),
               counts=torch.cat([load, load.new_tensor([n])]).to(torch.int32), prob=prob.detach(), lse=every)
    if c["train"]:
        out["dlogits"] = torch.autograd.grad(loss * s["dloss"].to(torch.float64).squeeze(), l)[0]
    return out


def _exact_distill(c, s):
    f64, tau = torch.float64, c["tau"]
    T, V = s["logits"].shape
    step = max(1, CHUNK // V)
    losses, grads = [], []
    for i in range(0, T, step):
        j = slice(i, min(T, i + step))
        z = s["logits"][j].to(f64).requires_grad_(True)
        logp = torch.log_softmax(z / tau, dim=1)
        kept = s["ids"][j] >= 0
        t = s["top"][j].to(f64) / tau
        t = t.masked_fill(~kept, -math.inf)
        logq = t - s["lse"][j].to(f64)[:, None] if c["lse"] else torch.log_softmax(t, dim=1)
        kd = torch.zeros(z.shape[0], dtype=f64, device=z.device)
        row, col = torch.nonzero(kept & (logq > -math.inf), as_tuple=True)
        lq = logq[row, col]
        kd = kd.index_add(0, row, torch.exp(lq) * (lq - logp[row, s["ids"][j][row, col].long()]))
        loss = s["kd_weight"] * tau ** 2 * kd
        if c["labels"]:
            lz = torch.log_softmax(z, dim=1)
            loss = loss - s["ce_weight"] * lz[torch.arange(z.shape[0], device=z.device), s["labels"][j].long()]
        loss = loss * s["weight"][j].to(f64)
        losses.append(loss.detach())
        if c["grad"]:
            grads.append(torch.autograd.grad(loss.sum(), z)[0])
    return dict(loss=torch.cat(losses), dlogits=torch.cat(grads) if c["grad"] else None)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "balance": _exact_balance, "distill": _exact_distill}[case["op"]](case, s)
