"""The training objective's operators in a run: router, balance loss, layer, likelihoods, and the gradients back to the router's
logits, against the same computation differentiated in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("gate", [0, 1, 2])
@pytest.mark.parametrize("T,kind", [(64, 0), (300, 1)])
def test_one_adaptation_step(gate, T, kind):
    from paper_2605_18643_b200 import inputs, zeda
    wl = inputs.tiny(seed=5, T=T)
    E, Z, K, d = wl.E, wl.Z, wl.K, wl.d
    alpha, w, V, eps = 0.05, 2.0, 777, 1e-6
    m = zeda.from_workload(wl, gate_mode=gate)
    x = wl.x.to(DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    vocab = (torch.randn(V, d, generator=g, device=DEV) / d ** 0.5).to(torch.bfloat16)
    target = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    target[: T // 4] = -100                                     # the prompt carries no likelihood
    padding = torch.ones(T, dtype=torch.bool, device=DEV)
    padding[-T // 8:] = False                                   # the batch's padding counts in neither loss
    target[~padding] = -100
    n_loss = int((target >= 0).sum())

    # forward
    logits = m.router_logits(x)
    r = m.route_from_logits(logits)
    balance, counts, p_mean, n = m.balance_loss(logits, r["topk_idx"], alpha, w, kind=kind, token_mask=padding)
    y = m.forward(x)
    h = zeda.residual_rmsnorm(y.clone(), None, eps=eps)
    lm = zeda.VocabLoss(vocab, T)
    nll, lse = lm.nll(h, target)
    loss = nll.sum() / n_loss + balance[0]
    # backward: likelihoods -> hidden states -> layer's output -> routing weights -> logits
    grad_nll = torch.full((T,), 1.0 / n_loss, device=DEV)
    grad_h, grad_vocab = lm.backward(h, target, nll, lse, grad_nll)
    yd = y.double()
    inv = torch.rsqrt((yd * yd).mean(dim=1, keepdim=True) + eps)
    gh = grad_h.double()
    grad_y = inv * (gh - yd * inv * inv * (gh * yd).mean(dim=1, keepdim=True))
    wgu, wd = wl.w_gate_up.to(DEV).double(), wl.w_down.to(DEV).double()
    xd = x.double()
    gu = torch.einsum("td,efd->tef", xd, wgu)
    He = wd.shape[2]
    out = torch.einsum("tef,edf->ted", torch.nn.functional.silu(gu[..., :He]) * gu[..., He:], wd)   # [T, E, d]
    zero = torch.zeros(T, Z, d, dtype=torch.float64, device=DEV)
    slots = torch.cat([out, zero], dim=1).gather(1, r["topk_idx"].long()[:, :, None].expand(-1, -1, d))
    grad_topk = (slots * grad_y[:, None, :]).sum(dim=2)
    grad_topk[~padding] = 0
    grad = m.router_backward(logits, r["topk_idx"], grad_topk_w=grad_topk.float(), grad_loss=torch.ones(1, device=DEV), counts=counts,
                             n_tokens=n, alpha=alpha, group_w=w, kind=kind, token_mask=padding)

    # the same, differentiated in 64 bits
    l = logits.double().requires_grad_()
    vd = vocab.double().requires_grad_()
    p = torch.softmax(l, dim=1)
    idx = r["topk_idx"].long()
    ps = p.gather(1, idx)
    if gate == zeda.GATE_SOFTMAX_RAW:
        wk = ps
    else:
        part = ps * (idx < E) if gate == zeda.GATE_RENORM_REAL else ps
        tot = part.sum(dim=1, keepdim=True)
        wk = part / torch.where(tot > 0, tot, torch.ones_like(tot))
    y64 = (wk[:, :, None] * slots).sum(dim=1)
    h64 = y64 * torch.rsqrt((y64 * y64).mean(dim=1, keepdim=True) + eps)
    live = target >= 0
    want_nll = torch.nn.functional.cross_entropy(h64[live] @ vd.t(), target[live].long(), reduction="sum") / n_loss
    keep = padding.double()[:, None]
    f = torch.nn.functional.one_hot(idx, E + Z).sum(dim=1).mul(keep).sum(dim=0) / keep.sum()
    P = (p * keep).sum(dim=0) / keep.sum()
    if kind == zeda.BALANCE_VANILLA:
        want_balance = alpha * (E + Z) / K * (f * P).sum()
    else:
        want_balance = alpha * (E + Z * w) / K * (f[:E].sum() * P[:E].sum() / E + f[E:].sum() * P[E:].sum() / (Z * w))
    want = want_nll + want_balance
    want.backward()
    # the layer's inner activations, its output, the hidden states and their gradient are each rounded to bf16 on the way (2^-9 rms
    # at most each), the output's error also through the norm: 8 such roundings
    tol = 8 * 2.0 ** -9
    assert abs(float(balance) - float(want_balance.detach())) <= 1e-5 * float(want_balance.detach())
    assert abs(float(loss) - float(want.detach())) <= tol * float(want.detach())
    for got, ref in ((grad.double(), l.grad), (grad_vocab.double(), vd.grad)):
        assert float((got - ref).norm()) <= tol * float(ref.norm())
    assert not grad[~padding].any()
    lm.check()
    m.last_counters()
    lm.close()
    m.close()
