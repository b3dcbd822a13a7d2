"""Timed cases of the training objective's operators: the losses of the adaptation stages with their gradients.

The objective adds two terms: the negative log likelihood of given tokens under a large vocabulary, and the
load-balancing loss of every router.  A case names one of four uses:

  balance      the balance loss with the per-candidate counts (ZedaMoE.balance_loss)
  router_step  the same and the gradient that reaches the router's logits: from the balance loss and from the
               routing weights, in one pass (ZedaMoE.router_backward)
  nll          a token's negative log likelihood from its hidden state and the vocabulary matrix, without the
               logits in memory (VocabLoss.nll)
  nll_step     the same and the gradients of hidden states and vocabulary matrix (VocabLoss.backward)

The routers are those of the benchmark (128 + 64 candidates, K 8; 64 + 32, K 4), of the tests' smallest layer
(8 + 4, K 2) and of the largest candidate count that a layer takes; hidden sizes are the layers' own.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
GATE_TOPK_NORM, GATE_SOFTMAX_RAW, GATE_RENORM_REAL = 0, 1, 2
GROUP, VANILLA = 0, 1  # of the balance loss: over the groups of normal and zero experts, over the candidates
IGNORED = -100  # a target of tokens that carry no loss
PLAIN_ROWS = 1024  # tokens whose logits the plain form holds at a time


def _router(name, use, T, E, Z, K, kind=GROUP, gate=GATE_TOPK_NORM, padding=0.0):
    c = dict(use=use, T=T, E=E, Z=Z, K=K, kind=kind, gate=gate, padding=padding)
    if name is not None:
        c["name"] = name
    return c


def _vocab(name, use, T, d, V, ignored=0.0):
    c = dict(use=use, T=T, d=d, V=V, ignored=ignored)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence's worth of tokens through the smallest layer: latency
        _router("balance_t64", "balance", 64, 8, 4, 2),
        # a packed training batch, the last sequences padded
        _router("balance_t8192", "balance", 8192, 128, 64, 8, padding=0.1),
        # the loss over a whole step's tokens, as many candidates as a layer takes but one, an odd number
        _router("balance_t65536", "balance", 65536, 320, 191, 8, kind=VANILLA),
        # a short sequence, raw softmax gates
        _router("router_step_t193", "router_step", 193, 64, 32, 4, gate=GATE_SOFTMAX_RAW),
        # the packed training batch with its gradient
        _router("router_step_t8192", "router_step", 8192, 128, 64, 8, padding=0.1),
        # the whole step's tokens, renormalised gates
        _router("router_step_t65536", "router_step", 65536, 320, 192, 8, kind=VANILLA, gate=GATE_RENORM_REAL),
        # the likelihood of one sampled token (the reward of one decoding step)
        _vocab("nll_t1", "nll", 1, 2048, 131072),
        # ragged sizes; the prompt's tokens carry no loss
        _vocab("nll_t777", "nll", 777, 1088, 32003, ignored=0.4),
        # teacher and student likelihoods of a training batch
        _vocab("nll_t8192", "nll", 8192, 2048, 131072, ignored=0.25),
        # a few tokens that carry loss, a large vocabulary: the vocabulary matrix and its gradient are what moves
        _vocab("nll_step_t64", "nll_step", 64, 2048, 65536),
        # ragged sizes
        _vocab("nll_step_t1001", "nll_step", 1001, 1088, 50021, ignored=0.4),
        # a training batch
        _vocab("nll_step_t8192", "nll_step", 8192, 2048, 131072, ignored=0.25),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    use = rng.choice(["balance", "router_step", "nll", "nll_step"])
    if use in ("balance", "router_step"):
        E, Z = _spread(rng, 2, 320), rng.choice([0, _spread(rng, 1, 192)])
        K = rng.randint(1, min(16, E + Z))
        return _router(None, use, _spread(rng, 1, 65536), E, Z, K, kind=rng.choice([GROUP, VANILLA]),
                       gate=rng.randint(0, 2), padding=rng.choice([0.0, 0.1, 0.5]))
    return _vocab(None, use, _spread(rng, 1, 8192), 64 * rng.randint(1, 32), _spread(rng, 500, 131072),
                  ignored=rng.choice([0.0, 0.25, 0.5]))


# ---------------------------------------------------------------------------------------- inputs
ALPHA, GROUP_W = 1e-2, 2.0


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE)

    s = dict(case)
    T = case["T"]
    if case["use"] in ("balance", "router_step"):
        E, Z, K = case["E"], case["Z"], case["K"]
        # a layer's logits: spread over a token's candidates, some candidates favoured
        s["logits"] = (randn(T, E + Z) + 0.5 * randn(E + Z)).contiguous()
        s["topk_idx"] = torch.topk(s["logits"], K, dim=1).indices.to(torch.int32).contiguous()
        s["mask"] = (rand(T) >= case["padding"]).to(torch.uint8) if case["padding"] else None
        s["grad_w"] = randn(T, K) / T
        s["grad_loss"] = torch.full((1,), 0.7, device=DEVICE)
        if own:
            from paper_2605_18643_b200 import zeda
            w = torch.zeros((E, 64, 64), dtype=torch.bfloat16, device=DEVICE)
            s["layer"] = zeda.ZedaMoE(torch.zeros((E + Z, 64), device=DEVICE), None,
                                      torch.zeros((E, 128, 64), dtype=torch.bfloat16, device=DEVICE), w, E, Z, K, T,
                                      gate_mode=case["gate"])
        return s
    d, V = case["d"], case["V"]
    s["w"] = (randn(V, d) * (0.9 / math.sqrt(d))).to(torch.bfloat16)
    said = torch.randint(0, V, (T,), generator=g, device=DEVICE)
    # hidden states as a final norm leaves them, leaning towards one token's row by a varying amount
    x = randn(T, d) + rand(T, 1) * 0.6 * math.sqrt(d) * torch.nn.functional.normalize(s["w"][said].float(), dim=1)
    s["x"] = (x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + 1e-6)).to(torch.bfloat16)
    other = torch.randint(0, V, (T,), generator=g, device=DEVICE)
    target = torch.where(rand(T) < 0.7, said, other)
    target[torch.randperm(T, generator=g, device=DEVICE)[:_ignored(case)]] = IGNORED
    s["target"] = target.to(torch.int32)
    # likelihoods weighted token by token, as rewards weight them
    s["grad_nll"] = (0.5 + rand(T)) / T
    if own:
        from paper_2605_18643_b200 import zeda
        s["loss"] = zeda.VocabLoss(s["w"], T, backward=case["use"] == "nll_step")
    return s


def _ignored(case):
    return int(case["T"] * case["ignored"])


# ----------------------------------------------------------------------------------------- a pass
def run(state):
    if state["use"] in ("balance", "router_step"):
        return _run_router(state) if own else _plain_router(state)
    return _run_vocab(state) if own else _plain_vocab(state)


def _run_router(s):
    m = s["layer"]
    loss, counts, p_mean, n_tokens = m.balance_loss(s["logits"], s["topk_idx"], ALPHA, GROUP_W, kind=s["kind"],
                                                    token_mask=s["mask"])
    if s["use"] == "balance":
        return loss, counts, p_mean, n_tokens
    grad = m.router_backward(s["logits"], s["topk_idx"], grad_topk_w=s["grad_w"], grad_loss=s["grad_loss"], counts=counts,
                             n_tokens=n_tokens, alpha=ALPHA, group_w=GROUP_W, kind=s["kind"], token_mask=s["mask"])
    return loss, counts, grad


def _run_vocab(s):
    nll, lse = s["loss"].nll(s["x"], s["target"])
    if s["use"] == "nll":
        return nll, lse
    grad_x, grad_w = s["loss"].backward(s["x"], s["target"], nll, lse, s["grad_nll"])
    return nll, grad_x, grad_w


def _plain_router(s):
    E, Z, K, T = s["E"], s["Z"], s["K"], s["T"]
    C = E + Z
    idx = s["topk_idx"].long()
    keep = s["mask"].bool() if s["mask"] is not None else torch.ones(T, dtype=torch.bool, device=DEVICE)
    z = s["logits"] - s["logits"].max(dim=1, keepdim=True).values
    e = torch.exp(z)
    p = e / e.sum(dim=1, keepdim=True)
    n_tokens = keep.sum().to(torch.int32).reshape(1)
    n = n_tokens.float().clamp(min=1)
    counts = torch.zeros(C, dtype=torch.int32, device=DEVICE)
    counts.index_add_(0, idx.reshape(-1), keep.to(torch.int32).repeat_interleave(K))
    f = counts.float() / n
    p_mean = (p * keep[:, None]).sum(dim=0) / n
    if s["kind"] == VANILLA:
        loss = ALPHA * C / K * (f * p_mean).sum()
        slope = ALPHA * C / K * f
    else:
        scale = ALPHA * (E + Z * GROUP_W) / K
        slope = torch.empty(C, device=DEVICE)
        slope[:E] = scale * f[:E].sum() / E
        loss = scale * f[:E].sum() * p_mean[:E].sum() / E
        if Z:
            slope[E:] = scale * f[E:].sum() / (Z * GROUP_W)
            loss = loss + scale * f[E:].sum() * p_mean[E:].sum() / (Z * GROUP_W)
    loss = loss.reshape(1)
    if s["use"] == "balance":
        return loss, counts, p_mean, n_tokens
    slope = slope * s["grad_loss"] / n
    grad = p * (slope - (p * slope).sum(dim=1, keepdim=True))
    gw = s["grad_w"]
    if s["gate"] == GATE_SOFTMAX_RAW:
        ps = torch.gather(p, 1, idx)
        grad = grad - p * (ps * gw).sum(dim=1, keepdim=True)
        grad.scatter_add_(1, idx, ps * gw)
    else:
        es = torch.gather(e, 1, idx)
        if s["gate"] == GATE_RENORM_REAL:
            es = torch.where(idx < E, es, torch.zeros_like(es))
        tot = es.sum(dim=1, keepdim=True)
        wk = torch.where(tot > 0, es / tot, torch.zeros_like(es))
        grad.scatter_add_(1, idx, wk * (gw - (wk * gw).sum(dim=1, keepdim=True)))
    return loss, counts, grad * keep[:, None]


def _plain_vocab(s):
    T, V = s["T"], s["V"]
    w = s["w"].float()
    nll = torch.zeros(T, device=DEVICE)
    lse = torch.zeros(T, device=DEVICE)
    step = s["use"] == "nll_step"
    if step:
        grad_x = torch.zeros((T, s["d"]), device=DEVICE)
        grad_w = torch.zeros((V, s["d"]), device=DEVICE)
    for t0 in range(0, T, PLAIN_ROWS):
        x = s["x"][t0:t0 + PLAIN_ROWS].float()
        target = s["target"][t0:t0 + PLAIN_ROWS].long()
        live = target >= 0
        label = target.clamp(min=0)[:, None]
        logits = x @ w.t()
        top = logits.max(dim=1, keepdim=True).values
        at_label = torch.gather(logits, 1, label)
        e = torch.exp(logits - top)
        den = e.sum(dim=1, keepdim=True)
        whole = top + torch.log(den)
        nll[t0:t0 + PLAIN_ROWS] = torch.where(live, (whole - at_label)[:, 0], torch.zeros_like(nll[:1]))
        lse[t0:t0 + PLAIN_ROWS] = torch.where(live, whole[:, 0], torch.zeros_like(nll[:1]))
        if step:
            g = torch.where(live, s["grad_nll"][t0:t0 + PLAIN_ROWS], torch.zeros_like(nll[:1]))[:, None]
            q = e / den
            q.scatter_add_(1, label, torch.full_like(at_label, -1.0))
            q = q * g
            grad_x[t0:t0 + PLAIN_ROWS] = q @ w
            grad_w += q.t() @ x
    if not step:
        return nll, lse
    return nll, grad_x.to(torch.bfloat16), grad_w.to(torch.bfloat16)


# ------------------------------------------------------------------------------------------- work
def work(case):
    T = case["T"]
    if case["use"] in ("balance", "router_step"):
        C, K = case["E"] + case["Z"], case["K"]
        # logits, ids and mask read once; per candidate a count and a mean; the step also reads the routing weights'
        # gradient and writes the logits'.  A maximum, an exponential, a sum and a division per logit, and as much again
        bytes_ = T * (4 * C + 4 * K + (1 if case["padding"] else 0)) + 8 * C
        if case["use"] == "balance":
            return {"bytes": bytes_, "flops": 5 * T * C}
        return {"bytes": bytes_ + T * (4 * C + 4 * K), "flops": 10 * T * C}
    d, V = case["d"], case["V"]
    live = T - _ignored(case)
    # tokens without loss are not read; the logits' product, and for the gradients two more (that a second product of
    # the logits takes the place of keeping them is not counted)
    if case["use"] == "nll":
        return {"bytes": 2 * d * (live + V) + 12 * T, "flops": 2 * live * d * V}
    return {"bytes": 2 * d * (live + V) + 2 * d * (T + V) + 16 * T, "flops": 6 * live * d * V}


# ------------------------------------------------------------------------- the definitions, 64 bits
def exact(case, seed):
    s = prepare(dict(case), seed)
    if case["use"] in ("balance", "router_step"):
        return _exact_router(s)
    return _exact_vocab(s)


def _exact_router(s):
    E, Z, K, T = s["E"], s["Z"], s["K"], s["T"]
    C = E + Z
    keep = torch.ones(T, dtype=torch.float64, device=DEVICE) if s["mask"] is None else s["mask"].double()
    l = s["logits"].double()
    p = torch.softmax(l, dim=1)
    n = float(keep.sum())
    chosen = torch.nn.functional.one_hot(s["topk_idx"].long(), C).sum(dim=1).double() * keep[:, None]  # [T, C]
    counts = chosen.sum(dim=0)
    f = counts / max(n, 1.0)
    P = (p * keep[:, None]).sum(dim=0) / max(n, 1.0)
    real = torch.arange(C, device=DEVICE) < E
    if s["kind"] == VANILLA:
        c = ALPHA * C / K * f
    else:
        share = torch.where(real, f[real].sum() / E, f[~real].sum() / (max(Z, 1) * GROUP_W))
        c = ALPHA * (E + Z * GROUP_W) / K * share
    loss = (c * P).sum().reshape(1)
    n_tokens = torch.tensor([int(n)], dtype=torch.int32, device=DEVICE)
    if s["use"] == "balance":
        return loss, counts.to(torch.int32), P, n_tokens
    # d loss / d p, through the softmax
    dp = keep[:, None] * (c * float(s["grad_loss"].double()) / max(n, 1.0))[None, :]
    slot = s["topk_idx"].long()
    gw = s["grad_w"].double()
    if s["gate"] == GATE_SOFTMAX_RAW:
        dp = dp.scatter_add(1, slot, keep[:, None] * gw)
    else:
        ps = torch.gather(p, 1, slot)
        if s["gate"] == GATE_RENORM_REAL:
            ps = ps * (slot < E)
        tot = ps.sum(dim=1, keepdim=True)
        inv = torch.where(tot > 0, 1.0 / tot, torch.zeros_like(tot))
        dps = inv * (gw - (gw * ps).sum(dim=1, keepdim=True) * inv)  # w_k = p_k / sum p
        if s["gate"] == GATE_RENORM_REAL:
            dps = dps * (slot < E)
        dp = dp.scatter_add(1, slot, keep[:, None] * dps)
    grad = p * (dp - (p * dp).sum(dim=1, keepdim=True))
    return loss, counts.to(torch.int32), grad


def _exact_vocab(s):
    T, V, d = s["T"], s["V"], s["d"]
    w = s["w"].double()
    rows = torch.nonzero(s["target"] >= 0)[:, 0]
    nll = torch.zeros(T, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(T, dtype=torch.float64, device=DEVICE)
    grad_x = torch.zeros((T, d), dtype=torch.float64, device=DEVICE)
    grad_w = torch.zeros((V, d), dtype=torch.float64, device=DEVICE)
    for part in rows.split(1024):
        x = s["x"][part].double()
        label = s["target"][part].long()
        logits = x @ w.t()
        whole = torch.logsumexp(logits, dim=1)
        own_logit = logits[torch.arange(len(part), device=DEVICE), label]
        lse[part] = whole
        nll[part] = whole - own_logit
        if s["use"] == "nll_step":
            q = torch.softmax(logits, dim=1)
            q[torch.arange(len(part), device=DEVICE), label] -= 1.0
            q *= s["grad_nll"][part].double()[:, None]
            grad_x[part] = q @ w
            grad_w += q.t() @ x
    if s["use"] == "nll":
        return nll, lse
    return nll, grad_x, grad_w
