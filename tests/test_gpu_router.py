"""Parity of the load balance loss and the gate's backward pass with the float64 oracle, on the GPU."""
import numpy as np
import pytest
import torch

import oracle as O
from oracle import operators_oracle as OO
from paper_2508_06024_amd import ec2moe as E
from paper_2508_06024_amd import workload as W
from tests.gpu_common import say

pytestmark = pytest.mark.gpu

DEV = "cuda"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def up(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def down(t):
    return t.double().cpu().numpy()


def _probs(rng, T, M, cand, sizes):
    """Gate probabilities in float32: random logits through the two softmaxes."""
    g = np.zeros((T, M))
    at, lg = 0, rng.normal(size=(T, len(sizes)))
    live = [[i for i in range(sum(sizes[:k]), sum(sizes[:k + 1])) if i in cand] for k in range(len(sizes))]
    lg[:, [k for k, m in enumerate(live) if not m]] = -np.inf
    pg = np.exp(lg - lg.max(axis=1, keepdims=True))
    pg /= pg.sum(axis=1, keepdims=True)
    for k, m in enumerate(live):
        if m:
            l = np.exp(rng.normal(size=(T, len(m))) * 1.5)
            g[:, m] = pg[:, k:k + 1] * l / l.sum(axis=1, keepdims=True)
    return g.astype(np.float32)


def _topk(g, k):
    return np.argsort(-g, axis=1, kind="stable")[:, :k].astype(np.int32)


# ----------------------------------------------------------------------------- balance loss

@pytest.mark.parametrize("T,M,k,pad", [
    (1, 1, 1, 0.0), (1, 8, 2, 0.0), (64, 8, 2, 0.3), (100, 7, 3, 0.0), (1000, 61, 5, 0.5), (4097, 64, 6, 0.0),
    (513, 256, 16, 0.2), (20000, 96, 8, 0.1), (70001, 256, 2, 0.0), (3, 255, 4, 0.0),
])
def test_balance_loss_matches_the_oracle(T, M, k, pad):
    say(f"balance_loss T={T} M={M} k={k} pad={pad}")
    rng = np.random.default_rng(T + M)
    g = _probs(rng, T, M, set(range(M)), [M])
    idx = _topk(g, k)
    valid = rng.random(T) >= pad if pad else None
    if valid is not None:
        g[~valid], idx[~valid] = np.nan, 1 << 30  # neither is read into anything
    loss, counts, d = E.balance_loss(up(g), up(idx, torch.int32), 0.01, None if valid is None else up(valid, torch.bool))
    ref = OO.balance_loss(np.where(np.isnan(g), 0, g).astype(np.float64), idx, 0.01, valid)
    np.testing.assert_array_equal(counts.cpu().numpy(), ref[1])
    # sums of at most 256 positive float32 terms in a row, the rest in float64; outputs rounded once,
    # the coefficient once
    np.testing.assert_allclose(down(loss)[0], ref[0], rtol=256 * 2.0 ** -24)
    np.testing.assert_allclose(down(d), ref[2], rtol=3 * 2.0 ** -24)


def test_balance_loss_without_valid_tokens_and_without_tokens():
    g = up(np.full((9, 8), 0.125))
    idx = torch.zeros((9, 2), dtype=torch.int32, device=DEV)
    for args in ((g, idx, 1.0, torch.zeros(9, dtype=torch.bool, device=DEV)), (g[:0], idx[:0], 1.0, None)):
        loss, counts, d = E.balance_loss(*args)
        assert float(loss) == 0 and (counts == 0).all() and (d == 0).all()


def test_balance_loss_outputs_are_optional():
    T, M, k = 3000, 16, 2
    rng = np.random.default_rng(0)
    g = up(_probs(rng, T, M, set(range(M)), [M]))
    idx = up(_topk(g.cpu().numpy(), k), torch.int32)
    full = E.balance_loss(g, idx, 2.0)
    desc = E.moe_desc(T, M, 1, 128, 128, k, E.BF16)
    ws = E.workspace(E.balance_loss_workspace_size(desc), DEV)
    loss = torch.empty(1, device=DEV)
    E.balance_loss_into(desc, g, idx, 2.0, loss, None, None, ws)
    assert torch.equal(loss, full[0])


# ----------------------------------------------------------------------------- gate backward

def _sizes(M, K, uneven, rng):
    if not uneven:
        return [M // K] * K
    cut = np.sort(rng.choice(np.arange(1, M), K - 1, replace=False)) if K > 1 else np.array([], int)
    return np.diff(np.concatenate([[0], cut, [M]])).astype(int).tolist()


def _check(name, got, ref, lim):
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), name
    assert (err <= lim).all(), f"{name}: worst excess {(err - lim).max():.3e} over a limit of {lim.flat[(err - lim).argmax()]:.3e}"


@pytest.mark.parametrize("T,d,M,K,k,keep,uneven,renorm,terms,pad,dtype", [
    (1, 128, 8, 2, 2, 8, False, True, "w", 0.0, torch.float32),
    (64, 128, 8, 2, 2, 6, False, True, "wb", 0.0, torch.float32),
    (17, 256, 9, 3, 3, 7, True, False, "wpb", 0.3, torch.bfloat16),
    (100, 384, 64, 8, 6, 48, False, True, "wb", 0.0, torch.bfloat16),
    (33, 128, 256, 64, 16, 200, True, True, "wpb", 0.2, torch.float32),
    (129, 128, 256, 16, 8, 256, False, True, "wb", 0.0, torch.bfloat16),
    (40, 256, 160, 160, 4, 100, False, True, "wp", 0.0, torch.bfloat16),
    (300, 640, 16, 4, 1, 9, True, False, "wb", 0.5, torch.bfloat16),
    (1000, 128, 12, 5, 2, 12, True, True, "p", 0.0, torch.float32),
    (515, 256, 40, 1, 4, 40, False, True, "wb", 0.0, torch.bfloat16),
    (2049, 128, 72, 8, 2, 50, True, True, "b", 0.1, torch.bfloat16),
])
def test_gate_backward_matches_the_oracle(T, d, M, K, k, keep, uneven, renorm, terms, pad, dtype):
    say(f"group_gate_backward T={T} d={d} M={M} K={K} k={k} {terms} {dtype}")
    rng = np.random.default_rng(T * 3 + M)
    sizes = _sizes(M, K, uneven, rng)
    groups = np.split(np.arange(M), np.cumsum(sizes)[:-1])
    groups = [g.tolist() for g in groups]
    cand = set(rng.choice(M, keep, replace=False).tolist())
    g = _probs(rng, T, M, cand, sizes)
    idx = _topk(g, k)
    valid = rng.random(T) >= pad if pad else None
    dw = rng.normal(size=(T, k)).astype(np.float32) if "w" in terms else None
    dp = (rng.normal(size=(T, M)) * 0.1).astype(np.float32) if "p" in terms else None
    db = rng.normal(size=M).astype(np.float32) if "b" in terms else None
    x = up(rng.normal(size=(T, d)), dtype)
    wg, wl = up(rng.normal(size=(K, d)) * 0.05, dtype), up(rng.normal(size=(M, d)) * 0.05, dtype)
    t = lambda a, ty=torch.float32: None if a is None else up(a, ty)
    call = lambda **kw: E.group_gate_backward(x, wg, wl, up(g), up(idx, torch.int32), t(dw), t(dp), t(db), t(valid, torch.bool),
                                              renormalize=renorm, group_sizes=sizes if uneven else None, **kw)
    got, g0 = call(), g.copy()
    dl, du, al, au = OO.gate_backward(g0.astype(np.float64), idx, groups, renorm, dw, dp, db, valid)
    X, WG, WL = down(x), down(wg), down(wl)
    # a logit's gradient is a sum of up to M + k float32 terms of magnitudes al; products and sums over
    # the M + K logits, or the T tokens, add a rounding each; x, W and the probabilities are exact
    e0 = (M + k + 24) * 2.0 ** -24
    el, eu = al * e0, au * e0
    if valid is not None:
        assert (down(got[0])[~valid] == 0).all()
        # whatever a padding token holds, it reaches nothing
        x[torch.from_numpy(~valid).to(DEV)] = float("nan")
        g[~valid] = np.inf
        assert all(torch.equal(u, v) for u, v in zip(got, call()))
        x[torch.from_numpy(~valid).to(DEV)] = 0
    ref = dl @ WL + du @ WG
    _check("d_x", down(got[0]), ref, (el + al * (M + K) * 2.0 ** -24) @ np.abs(WL) + (eu + au * (M + K) * 2.0 ** -24) @ np.abs(WG)
           + np.abs(ref) * HALF[dtype] + 1e-37)
    eT = (T + 16) * 2.0 ** -24
    _check("d_w_global", down(got[1]), du.T @ X, (eu + au * eT).T @ np.abs(X) + 1e-37)
    _check("d_b_global", down(got[2]), du.sum(axis=0), (eu + au * eT).sum(axis=0) + 1e-37)
    _check("d_w_local", down(got[3]), dl.T @ X, (el + al * eT).T @ np.abs(X) + 1e-37)
    _check("d_b_local", down(got[4]), dl.sum(axis=0), (el + al * eT).sum(axis=0) + 1e-37)
    off = [e for e in range(M) if e not in cand]
    assert (down(got[3])[off] == 0).all() and (down(got[4])[off] == 0).all()
    again = call()
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    no_dx = call(with_dx=False)
    assert no_dx[0] is None and all(torch.equal(a, b) for a, b in zip(got[1:], no_dx[1:]))


@pytest.mark.parametrize("renorm", [True, False])
def test_gate_backward_of_repeated_and_missing_selections(renorm):
    """A token may name an expert twice (its gradients add), and an id outside [0, M) selects nothing."""
    rng = np.random.default_rng(15)
    T, d, M, K, k = 70, 128, 16, 4, 4
    g = _probs(rng, T, M, set(range(M)), [4] * 4)
    idx = _topk(g, k)
    idx[:, 3] = idx[:, 0]
    dw = rng.normal(size=(T, k)).astype(np.float32)
    x, wg, wl = (up(rng.normal(size=(n, d)) * 0.3) for n in (T, K, M))
    groups = [list(range(4 * i, 4 * i + 4)) for i in range(K)]
    X, WG, WL = down(x), down(wg), down(wl)

    def check(got, sel, dw):
        dl, du, al, au = (np.zeros((T, n)) for n in (M, K, M, K))
        for t in range(T):  # the oracle takes selections of one length
            keep = (sel[t] >= 0) & (sel[t] < M)
            o = OO.gate_backward(g[t:t + 1].astype(np.float64), sel[t:t + 1, keep], groups, renorm, dw[t:t + 1, keep])
            dl[t], du[t], al[t], au[t] = (a[0] for a in o)
        e0 = (M + k + 24) * 2.0 ** -24
        eX, eT = e0 + (M + K + 1) * 2.0 ** -24, e0 + (T + 16) * 2.0 ** -24
        _check("d_x", down(got[0]), dl @ WL + du @ WG, eX * (al @ np.abs(WL) + au @ np.abs(WG)) + 1e-37)
        _check("d_w_global", down(got[1]), du.T @ X, eT * (au.T @ np.abs(X)) + 1e-37)
        _check("d_w_local", down(got[3]), dl.T @ X, eT * (al.T @ np.abs(X)) + 1e-37)

    call = lambda sel: E.group_gate_backward(x, wg, wl, up(g), up(sel, torch.int32), up(dw), renormalize=renorm)
    check(call(idx), idx, dw)
    idx[:, 1] = np.where(np.arange(T) % 2, -1, M + 5)
    check(call(idx), idx, dw)


def test_gate_backward_refuses_pruned_groups():
    x, wg, wl = (torch.zeros((n, 128), device=DEV) for n in (4, 2, 8))
    g, idx = torch.full((4, 8), 0.125, device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(E.Ec2moeError):
        E.group_gate_backward(x, wg, wl, g, idx, top_groups=1)
    assert E.group_gate_backward(x, wg, wl, g, idx, top_groups=2)[0].abs().sum() == 0


def test_gate_backward_of_one_renormalised_selection_is_zero():
    rng = np.random.default_rng(4)
    g = _probs(rng, 50, 8, set(range(8)), [4, 4])
    x = up(rng.normal(size=(50, 128)), torch.bfloat16)
    w = lambda n: up(rng.normal(size=(n, 128)), torch.bfloat16)
    out = E.group_gate_backward(x, w(2), w(8), up(g), up(_topk(g, 1), torch.int32), d_topk_w=up(rng.normal(size=(50, 1))))
    assert all((o == 0).all() for o in out)


def test_gate_backward_without_tokens_writes_zeros():
    x = torch.empty((0, 128), device=DEV)
    w = lambda n: torch.ones((n, 128), device=DEV)
    out = E.group_gate_backward(x, w(2), w(8), torch.empty((0, 8), device=DEV), torch.empty((0, 2), dtype=torch.int32, device=DEV),
                                d_balance=torch.ones(8, device=DEV))
    assert out[0].shape == (0, 128) and all((o == 0).all() for o in out[1:])


def test_router_step_gradients_are_the_differences_of_its_loss():
    """Gate, balance loss and gate backward together, as a training step of the router calls them:
    the gradients of sum(c topk_w) + balance loss against central differences of the oracle's gate
    (selection and counts held, as in the definition)."""
    rng = np.random.default_rng(11)
    T, d, M, K, k = 12, 128, 8, 2, 3
    words = W.mask_words([0, 1, 2, 4, 5, 7], M)
    x, wg, wl = rng.normal(size=(T, d)), rng.normal(size=(K, d)) * 0.1, rng.normal(size=(M, d)) * 0.1
    x, wg, wl = (np.float64(np.float32(a)) for a in (x, wg, wl))
    bg, bl = np.float64(np.float32(rng.normal(size=K) * 0.1)), np.float64(np.float32(rng.normal(size=M) * 0.1))
    c = np.float32(rng.normal(size=(T, k)))
    valid = np.arange(T) % 5 != 3
    idx, w, probs = E.gate(up(x), words, up(wg), up(bg), up(wl), up(bl), K, k, with_probs=True)
    loss, counts, d_bal = E.balance_loss(probs, idx, 0.5, up(valid, torch.bool))
    got = E.group_gate_backward(up(x), up(wg), up(wl), probs, idx, up(c), None, d_bal, up(valid, torch.bool))
    sel, cnt = idx.cpu().numpy(), counts.cpu().numpy()

    def f(x, wg, bg, wl, bl):
        g = O.group_gate_probs(x, wg, bg, wl, bl, words, K)
        total = 0.0
        for t in np.nonzero(valid)[0]:
            s = g[t, sel[t]]
            total += float(c[t] @ (s / s.sum()))
        n = valid.sum()
        return total + 0.5 * M * float((cnt / (n * k)) @ (g[valid].sum(axis=0) / n))

    base = [x, wg, bg, wl, bl]
    h = 1e-5
    for which, grad in zip(range(5), got):
        grad = down(grad)
        for _ in range(12):
            at = tuple(rng.integers(0, n) for n in base[which].shape)
            lo, hi = [b.copy() for b in base], [b.copy() for b in base]
            lo[which][at] -= h
            hi[which][at] += h
            diff = (f(*hi) - f(*lo)) / (2 * h)
            # float32 probabilities from the gate: 1e-5 of the largest, differences themselves 1e-9
            assert abs(diff - grad[at]) <= 1e-4 * np.abs(grad).max() + 1e-8, (which, at, diff, grad[at])


def test_router_operators_captured_in_a_graph():
    rng = np.random.default_rng(12)
    T, d, M, K, k = 5000, 256, 32, 4, 2
    desc = E.moe_desc(T, M, K, d, 128, k, torch.bfloat16)
    wg, wl = up(rng.normal(size=(K, d)) * 0.05, torch.bfloat16), up(rng.normal(size=(M, d)) * 0.05, torch.bfloat16)
    xs = [up(rng.normal(size=(T, d)), torch.bfloat16) for _ in range(2)]
    words = W.mask_words(list(range(M)), M)
    dw = up(rng.normal(size=(T, k)))
    new = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device=DEV)
    x, idx, w, probs = xs[0].clone(), new(T, k, dt=torch.int32), new(T, k), new(T, M)
    loss, counts, bal = new(1), new(M, dt=torch.int32), new(M)
    out = dict(d_x=torch.empty_like(x), d_w_global=new(K, d), d_b_global=new(K), d_w_local=new(M, d), d_b_local=new(M))
    ws1, ws2 = E.workspace(E.balance_loss_workspace_size(desc), DEV), E.workspace(E.gate_backward_workspace_size(desc), DEV)

    def step():
        E.group_gate_ex(desc, None, words, x, wg, None, wl, None, idx, w, probs)
        E.balance_loss_into(desc, probs, idx, 0.01, loss, counts, bal, ws1)
        E.group_gate_backward_into(desc, None, x, wg, wl, probs, idx, ws2, d_topk_w=dw, d_balance=bal, **out)

    held = lambda: [t.clone() for t in (loss, counts, bal, *out.values())]
    refs = []
    for v in xs:
        x.copy_(v)
        step()
        refs.append(held())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(5):
        x.copy_(xs[rep % 2])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held(), refs[rep % 2])), f"replay {rep}"
        x.copy_(xs[1 - rep % 2])
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held(), refs[1 - rep % 2]))


def test_binding_refuses_wrong_operands():
    g, idx = torch.full((4, 8), 0.125, device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    x, wg, wl = (torch.zeros((n, 128), device=DEV) for n in (4, 2, 8))
    with pytest.raises(TypeError):
        E.balance_loss(g.double(), idx)
    with pytest.raises(TypeError):
        E.balance_loss(g, idx.long())
    with pytest.raises(TypeError):
        E.balance_loss(g, idx, token_valid=torch.ones(4, device=DEV))
    with pytest.raises(ValueError):
        E.balance_loss(g, idx, token_valid=torch.ones(5, dtype=torch.bool, device=DEV))
    with pytest.raises(ValueError):
        E.group_gate_backward(x, wg, wl, g, idx, d_topk_w=torch.zeros((4, 3), device=DEV))
    with pytest.raises(ValueError):
        E.group_gate_backward(x, wg, wl, g.t().contiguous().t(), idx)
    with pytest.raises(E.Ec2moeError):
        E.group_gate_backward(x, wg, wl, g, idx, group_sizes=[3, 4])
    assert E.group_gate_backward(x, wg, wl, g, idx)[1].abs().sum() == 0  # no gradient given: zeros
