"""Balance loss with counts, and the gradient to the router's logits, against a plain implementation in 64 bits.

Tolerances.  A probability of the kernels is an fp32 exponential (2 ulp) of a rounded difference (half an ulp of up to 20, so
1.2e-6 relative at the far end), times a rounded reciprocal of a sum of up to 512 such terms (warp tree: 9 + 16 additions of
2^-24): below 4e-6 relative.  A mean over T tokens adds at most T / (CTAs x warps) + 40 additions of positive terms to that
(below 100 here: 6e-6).  Gradients are differences of such products: 1.2e-5 of the sum of the magnitudes that they are made of.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P_RTOL, GRAD_TOL = 1e-5, 1.2e-5


def layer(zeda, E, Z, K, T, gate=0, flags=0):
    return zeda.ZedaMoE(torch.zeros((E + Z, 64), device=DEV), None, torch.zeros((E, 128, 64), dtype=torch.bfloat16, device=DEV),
                        torch.zeros((E, 64, 64), dtype=torch.bfloat16, device=DEV), E, Z, K, max(T, 1), gate_mode=gate, flags=flags)


def batch(T, C, K, seed, masked=0.0):
    rng = np.random.default_rng(seed)
    logits = (rng.standard_normal((T, C)) * 2 + rng.standard_normal(C)).astype(np.float32)
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :K].astype(np.int32)
    mask = (rng.random(T) >= masked).astype(np.uint8) if masked else None
    return logits, idx, mask


def ref_loss(logits, idx, mask, E, Z, K, kind, alpha, w):
    """(loss, counts, P, n, slopes): the slopes are dL/dP_i."""
    T, C = logits.shape
    keep = np.ones(T, bool) if mask is None else mask != 0
    l = logits[keep].astype(np.float64)
    top = l.max(axis=1, keepdims=True, initial=-np.inf)
    e = np.exp(l - np.where(np.isfinite(top), top, 0.0))
    den = e.sum(axis=1, keepdims=True)
    p = np.divide(e, den, out=np.zeros_like(e), where=den != 0)
    n = int(keep.sum())
    chosen = idx[keep].ravel()
    counts = np.bincount(chosen[(chosen >= 0) & (chosen < C)], minlength=C)
    f = counts / max(n, 1)
    P = p.sum(axis=0) / max(n, 1)
    if kind == 1:
        s = alpha * C / K * f
    else:
        s = np.empty(C)
        scale = alpha * (E + Z * w) / K
        s[:E] = scale * f[:E].sum() / E
        if Z:
            s[E:] = scale * f[E:].sum() / (Z * w)
    return float((s * P).sum()), counts, P, n, s


def ref_grad(logits, idx, mask, E, K, gate, slopes, n, grad_loss, grad_w):
    """(gradient, sum of the magnitudes it is made of)"""
    T, C = logits.shape
    keep = np.ones(T, bool) if mask is None else mask != 0
    out, mag = np.zeros((T, C)), np.zeros((T, C))
    for t in np.nonzero(keep)[0]:
        l = logits[t].astype(np.float64)
        m = l.max()
        e = np.exp(l - (m if np.isfinite(m) else 0.0))
        p = e / e.sum() if e.sum() else e
        if grad_loss is not None:
            s = slopes * (float(grad_loss) / max(n, 1))
            s = s - s[0]
            out[t] += p * (s - (p * s).sum())
            mag[t] += p * (np.abs(s) + (p * np.abs(s)).sum())
        if grad_w is not None:
            g = grad_w[t].astype(np.float64)
            ids = idx[t]
            ok = (ids >= 0) & (ids < (E if gate == 2 else C))
            if not ok.any():
                continue
            lk = l[ids[ok]]
            if gate == 1:
                pk = p[ids[ok]]
                np.add.at(out[t], ids[ok], pk * g[ok])
                out[t] -= p * (pk * g[ok]).sum()
                np.add.at(mag[t], ids[ok], pk * np.abs(g[ok]))
                mag[t] += p * (pk * np.abs(g[ok])).sum()
            elif np.isfinite(lk.max()):
                wk = np.exp(lk - lk.max())
                wk /= wk.sum()
                np.add.at(out[t], ids[ok], wk * (g[ok] - (wk * g[ok]).sum()))
                np.add.at(mag[t], ids[ok], wk * (np.abs(g[ok]) + (wk * np.abs(g[ok])).sum()))
    return out, mag


def cu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


SHAPES = [  # T, E, Z, K, masked
    (1, 1, 0, 1, 0.0), (1, 8, 4, 2, 0.0), (64, 8, 4, 2, 0.3), (33, 31, 1, 3, 0.0), (777, 64, 32, 4, 0.2), (1001, 60, 5, 16, 0.5),
    (2500, 100, 28, 6, 0.0), (4099, 128, 64, 8, 0.1), (300, 129, 64, 8, 0.0), (6000, 200, 57, 8, 0.1), (700, 320, 192, 16, 0.0),
    (5000, 257, 254, 5, 0.9), (130, 512, 0, 2, 0.0),
]


@pytest.mark.parametrize("T,E,Z,K,masked", SHAPES)
@pytest.mark.parametrize("kind", [0, 1])
def test_balance_loss_and_counts(T, E, Z, K, masked, kind):
    from paper_2605_18643_b200 import zeda
    logits, idx, mask = batch(T, E + Z, K, seed=T + kind, masked=masked)
    m = layer(zeda, E, Z, K, T)
    want = ref_loss(logits, idx, mask, E, Z, K, kind, 0.013, 2.0)
    got = [None, None]
    for i in range(2):
        got[i] = [t.cpu().numpy() for t in m.balance_loss(cu(logits), cu(idx), 0.013, 2.0, kind=kind, token_mask=cu(mask))]
        loss, counts, p, n = got[i]
        assert n[0] == want[3] and np.array_equal(counts, want[1])
        assert np.allclose(p, want[2], rtol=P_RTOL, atol=1e-30)
        assert np.allclose(loss, want[0], rtol=P_RTOL, atol=0)
    assert all(np.array_equal(a, b) for a, b in zip(*got))
    m.close()


@pytest.mark.parametrize("T,E,Z,K,masked", SHAPES)
@pytest.mark.parametrize("gate", [0, 1, 2])
@pytest.mark.parametrize("parts", ["both", "balance", "gate"])
def test_router_gradient(T, E, Z, K, masked, gate, parts):
    from paper_2605_18643_b200 import zeda
    kind = (T + gate) % 2
    logits, idx, mask = batch(T, E + Z, K, seed=2 * T + gate, masked=masked)
    rng = np.random.default_rng(T)
    gw = (rng.standard_normal((T, K)) / T).astype(np.float32) if parts != "balance" else None
    gl = np.float32(0.7) if parts != "gate" else None
    _, counts, _, n, s = ref_loss(logits, idx, mask, E, Z, K, kind, 0.013, 2.0)
    want, mag = ref_grad(logits, idx, mask, E, K, gate, s, n, gl, gw)
    m = layer(zeda, E, Z, K, T, gate)
    kw = dict(kind=kind, alpha=0.013, group_w=2.0, token_mask=cu(mask))
    if gl is not None:
        kw.update(grad_loss=torch.full((1,), float(gl), device=DEV), counts=cu(counts.astype(np.int32)),
                  n_tokens=torch.tensor([n], dtype=torch.int32, device=DEV))
    got = m.router_backward(cu(logits), cu(idx), grad_topk_w=cu(gw), out=torch.full((T, E + Z), float("nan"), device=DEV), **kw)
    err = np.abs(got.cpu().numpy() - want)
    assert np.all(err <= GRAD_TOL * mag + 1e-38)
    assert torch.equal(got, m.router_backward(cu(logits), cu(idx), grad_topk_w=cu(gw), **kw))
    m.close()


@pytest.mark.parametrize("kind", [0, 1])
def test_the_gradient_is_the_loss_s_difference_quotient(kind):
    from paper_2605_18643_b200 import zeda
    T, E, Z, K, h = 40, 24, 12, 4, 2.0 ** -4
    logits, idx, _ = batch(T, E + Z, K, seed=3)
    rng = np.random.default_rng(4)
    m = layer(zeda, E, Z, K, T)
    loss, counts, _, n = m.balance_loss(cu(logits), cu(idx), 1.0, 2.0, kind=kind)
    g = m.router_backward(cu(logits), grad_loss=torch.ones(1, device=DEV), counts=counts, n_tokens=n, alpha=1.0, group_w=2.0, kind=kind)
    s = ref_loss(logits, idx, None, E, Z, K, kind, 1.0, 2.0)[4]
    for _ in range(4):
        v = rng.uniform(-1, 1, logits.shape)
        at = [float(m.balance_loss(cu((logits + d * v).astype(np.float32)), cu(idx), 1.0, 2.0, kind=kind)[0]) for d in (h, -h)]
        want = (g.cpu().numpy().astype(np.float64) * v).sum()
        # a loss is the mean of E_p[s]; its third derivative along |v| <= 1 is a joint cumulant of s and three v, at most
        # 19 max|s|; the losses are off by P_RTOL, the logits by half a step of up to 8
        tol = h * h / 6 * 19 * np.abs(s).max() + (2 * P_RTOL * float(loss) + 2 * 2.0 ** -21 * np.abs(s).max()) / (2 * h)
        assert abs((at[0] - at[1]) / (2 * h) - want) <= tol
        assert tol < 0.2 * np.abs(s).max()
    m.close()


def test_masked_tokens_are_not_read_and_get_zeros():
    from paper_2605_18643_b200 import zeda
    T, E, Z, K = 100, 16, 8, 2
    logits, idx, _ = batch(T, E + Z, K, seed=5)
    mask = np.ones(T, np.uint8)
    mask[::3] = 0
    clean = logits.copy()
    logits[::3] = np.nan
    logits[3::6] = np.inf
    idx_bad = idx.copy()
    idx_bad[::3] = 2 ** 30
    m = layer(zeda, E, Z, K, T)
    gw = torch.randn(T, K, device=DEV)
    outs = []
    for l, i in ((logits, idx_bad), (clean, idx)):
        loss, counts, p, n = m.balance_loss(cu(l), cu(i), 0.1, 2.0, token_mask=cu(mask).bool())
        g = m.router_backward(cu(l), cu(i), grad_topk_w=gw, grad_loss=torch.ones(1, device=DEV), counts=counts, n_tokens=n, alpha=0.1,
                              group_w=2.0, token_mask=cu(mask))
        outs.append((loss, counts, p, n, g))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert not outs[0][4][::3].any() and outs[0][4].isfinite().all()
    # nothing counts at all
    none = torch.zeros(T, dtype=torch.uint8, device=DEV)
    loss, counts, p, n = m.balance_loss(cu(logits), cu(idx_bad), 0.1, 2.0, token_mask=none)
    assert not loss.any() and not counts.any() and not p.any() and not n.any()
    g = m.router_backward(cu(logits), cu(idx_bad), grad_topk_w=gw, grad_loss=torch.ones(1, device=DEV), counts=counts, n_tokens=n,
                          alpha=0.1, group_w=2.0, token_mask=none)
    assert not g.any()
    m.close()


@pytest.mark.parametrize("gate", [0, 1, 2])
def test_infinite_logits_padding_slots_and_an_id_that_comes_twice(gate):
    from paper_2605_18643_b200 import zeda
    T, E, Z, K = 70, 20, 13, 5
    logits, idx, _ = batch(T, E + Z, K, seed=6)
    logits[3] = -np.inf                       # a token with nothing to choose from
    logits[4, 5:] = -np.inf                   # candidates that are closed
    logits[5] = np.finfo(np.float32).min      # masked by the type's lowest value: all alike
    logits[6, ::2] = np.finfo(np.float32).min
    idx[7] = -1
    idx[8, 2:] = [-5, E + Z, 2 ** 31 - 1]
    idx[9] = [4, 4, 4, 17, 17]
    idx[10] = [E, E + 1, E + 2, E + 3, E + 4]  # zero experts only
    idx[11] = 2
    gw = np.random.default_rng(7).standard_normal((T, K)).astype(np.float32)
    m = layer(zeda, E, Z, K, T, gate)
    for kind in (0, 1):
        want = ref_loss(logits, idx, None, E, Z, K, kind, 0.5, 3.0)
        loss, counts, p, n = m.balance_loss(cu(logits), cu(idx), 0.5, 3.0, kind=kind)
        assert np.array_equal(counts.cpu().numpy(), want[1]) and int(n) == T
        assert np.allclose(p.cpu().numpy(), want[2], rtol=P_RTOL, atol=1e-30) and np.allclose(float(loss), want[0], rtol=P_RTOL)
        g, mag = ref_grad(logits, idx, None, E, K, gate, want[4], T, 1.5, gw)
        got = m.router_backward(cu(logits), cu(idx), grad_topk_w=cu(gw), grad_loss=torch.full((1,), 1.5, device=DEV), counts=counts,
                                n_tokens=n, alpha=0.5, group_w=3.0, kind=kind).cpu().numpy()
        assert np.all(np.abs(got - g) <= GRAD_TOL * mag + 1e-38)
    # a NaN stays in its token
    logits[20, 3] = np.nan
    got = m.router_backward(cu(logits), cu(idx), grad_topk_w=cu(gw)).cpu().numpy()
    rest = np.arange(T) != 20
    assert np.isfinite(got[rest]).all()
    assert np.isnan(float(m.balance_loss(cu(logits), cu(idx), 0.5, 3.0)[0]))
    m.close()


def test_counts_of_several_calls_give_the_whole_batch_s_gradient():
    from paper_2605_18643_b200 import zeda
    T, E, Z, K = 500, 32, 16, 4
    logits, idx, mask = batch(T, E + Z, K, seed=8, masked=0.2)
    m = layer(zeda, E, Z, K, T)
    one = torch.ones(1, device=DEV)
    kw = dict(grad_loss=one, alpha=0.3, group_w=2.0, kind=1)
    whole = m.balance_loss(cu(logits), cu(idx), 0.3, 2.0, kind=1, token_mask=cu(mask))
    want = m.router_backward(cu(logits), counts=whole[1], n_tokens=whole[3], token_mask=cu(mask), **kw)
    cut = 193
    parts = [m.balance_loss(cu(logits[a:b]), cu(idx[a:b]), 0.3, 2.0, kind=1, token_mask=cu(mask[a:b])) for a, b in ((0, cut), (cut, T))]
    counts, n = parts[0][1] + parts[1][1], parts[0][3] + parts[1][3]
    got = [m.router_backward(cu(logits[a:b]), counts=counts, n_tokens=n, token_mask=cu(mask[a:b]), **kw) for a, b in ((0, cut), (cut, T))]
    assert torch.equal(torch.cat(got), want)
    m.close()


@pytest.mark.parametrize("flags", [0, 4])
def test_calls_in_a_row_in_a_graph_and_on_another_stream(flags):
    from paper_2605_18643_b200 import zeda
    E, Z, K = 128, 64, 8
    m = layer(zeda, E, Z, K, 4096, flags=flags)
    sets = [batch(T, E + Z, K, seed=T, masked=0.1) for T in (4096, 64, 1500)]
    dev = [(cu(l), cu(i), cu(k)) for l, i, k in sets]
    one = torch.ones(1, device=DEV)

    def step(l, i, k):
        loss, counts, p, n = m.balance_loss(l, i, 0.01, 2.0, token_mask=k)
        return loss, counts, p, n, m.router_backward(l, i, grad_topk_w=torch.ones(l.shape[0], K, device=DEV), grad_loss=one, counts=counts,
                                                     n_tokens=n, alpha=0.01, group_w=2.0, token_mask=k)

    alone = []
    for d in dev:
        alone.append([t.clone() for t in step(*d)])
        torch.cuda.synchronize()
    for _ in range(3):
        for got, want in zip([step(*d) for d in dev], alone):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(*dev[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, alone[1]))
    # captured once, replayed on new contents of the same buffers
    l, i, k = (t.clone() for t in dev[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step(l, i, k)
    for src in (dev[2], [t[:1500].clone() for t in dev[0]], dev[2]):
        for dst, t in zip((l, i, k), src):
            dst.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, step(*src)))
    m.close()


def test_agrees_with_the_framework_s_routing_and_statistics():
    from paper_2605_18643_b200 import inputs, zeda
    wl = inputs.tiny(seed=3, T=200)
    m = zeda.from_workload(wl)
    x = wl.x.to(DEV)
    f, p, o = m.stats(x)
    logits = m.router_logits(x)
    r = m.route(x)
    loss, counts, pm, n = m.balance_loss(logits, r["topk_idx"], 1.0, 2.0)
    assert torch.equal(counts[:wl.E], r["counts"]) and int(n) == 200
    assert torch.allclose(counts / 200, f, rtol=2e-7, atol=0) and torch.allclose(pm, p, rtol=2 * P_RTOL)
    want = (wl.E + 2.0 * wl.Z) / wl.K * (float(o[2]) / wl.E + float(o[3]) / (wl.Z * 2.0))
    assert abs(float(loss) - want) <= 3 * P_RTOL * want
    # the routing kept in the handle is still the last call's
    assert torch.equal(m.token_zero_share(200), (r["topk_idx"] >= wl.E).float().sum(dim=1) / wl.K)
    m.close()


def test_refusals():
    from paper_2605_18643_b200 import zeda
    T, E, Z, K = 16, 8, 4, 2
    m = layer(zeda, E, Z, K, T)
    logits, idx, _ = batch(T, E + Z, K, seed=1)
    l, i = cu(logits), cu(idx)
    for bad in (dict(kind=2), dict(alpha=float("nan")), dict(alpha=float("inf")), dict(group_w=0.0), dict(group_w=-1.0),
                dict(group_w=float("nan"))):
        kw = dict(alpha=0.1, group_w=2.0, kind=0)
        kw.update(bad)
        with pytest.raises(zeda.ZedaError) as e:
            m.balance_loss(l, i, **kw)
        assert e.value.status == zeda.ERR_INVALID_ARG
    with pytest.raises(zeda.ZedaError):
        m.router_backward(l, i)                                            # no gradient at all
    with pytest.raises(zeda.ZedaError):
        m.router_backward(l, grad_loss=torch.ones(1, device=DEV), alpha=0.1)   # no counts
    with pytest.raises(zeda.ZedaError):
        m.router_backward(l, grad_topk_w=torch.ones(T, K, device=DEV))     # no ids
    with pytest.raises(zeda.ZedaError):
        m.router_backward(l, i, grad_topk_w=torch.ones(T, K, device=DEV), out=l)   # in place
    big = torch.zeros((T + 1, E + Z), device=DEV)
    with pytest.raises(zeda.ZedaError):
        m.balance_loss(big, torch.zeros((T + 1, K), dtype=torch.int32, device=DEV), 0.1)
    # no tokens: nothing happens
    loss, counts, p, n = m.balance_loss(l[:0], i[:0], 0.1)
    assert not loss.any() and not counts.any() and not n.any()
    assert m.router_backward(l[:0], i[:0], grad_topk_w=torch.ones(0, K, device=DEV)).shape == (0, E + Z)
    m.last_counters()
    m.close()
