"""CPU oracle of the 8-bit expert products and of the router's training operators: plain NumPy
float64 from the definitions, sharing no code with the HIP library.

TEST INFRASTRUCTURE, NOT PRODUCT CODE.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128


# ----------------------------------------------------------------------------- 8-bit numbers

def e4m3_values():
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; no
    infinity, NaN where all seven lower bits are set."""
    out = np.empty(256)
    for c in range(256):
        sign, e, m = (-1.0 if c & 0x80 else 1.0), (c >> 3) & 15, c & 7
        out[c] = sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        if (c & 0x7f) == 0x7f:
            out[c] = np.nan
    return out


_POSITIVE = e4m3_values()[:127]  # ascending: 0 .. 448


def e4m3_round(v):
    """Nearest representable value, ties to the even code; beyond 448 the largest."""
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    pick = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(_POSITIVE[pick], v)


def e4m3_step(v):
    """Distance of the two representable values around |v|, and of |v| to their midpoint."""
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    step = _POSITIVE[hi] - _POSITIVE[hi - 1]
    # the midpoint nearest to a: inside its own interval, or just across a representable value
    mids = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2
    at = np.clip(np.searchsorted(mids, a), 1, mids.size - 1)
    return step, np.minimum(np.abs(a - mids[at - 1]), np.abs(a - mids[at]))


def block_amax(x, block_rows):
    """Largest magnitude of each block_rows x 128 block of x [rows][cols], at least 2^-100."""
    rows, cols = x.shape
    nb = -(-rows // block_rows)
    out = np.empty((nb, cols // BLOCK))
    for i in range(nb):
        for j in range(cols // BLOCK):
            blk = x[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            out[i, j] = max(np.abs(blk).max(), 2.0 ** -100)
    return out


def spread(blocks, rows, block_rows):
    """A value per block as one per element."""
    return np.repeat(np.repeat(blocks, block_rows, axis=0)[:rows], BLOCK, axis=1)


def fp8_quantize(x, block_rows):
    """(values of the codes, scales) of x [rows][cols]."""
    x = np.asarray(x, np.float64)
    amax = block_amax(x, block_rows)
    return e4m3_round(448.0 * x / spread(amax, x.shape[0], block_rows)), amax / 448.0


def fp8_numbers(q, scale, block_rows):
    """What codes (given as values) and scales stand for."""
    return np.asarray(q, np.float64) * spread(np.asarray(scale, np.float64), q.shape[0], block_rows)


def fp8_matmul(a, w, seg, out):
    """out[p] = a[p] w_e^T for the rows of every segment, on numbers; (out, sum of |products|)."""
    out = np.array(out, np.float64)
    size = np.zeros_like(out)
    for e in range(len(w)):
        s = slice(int(seg[e]), int(seg[e + 1]))
        out[s] = a[s] @ w[e].T
        size[s] = np.abs(a[s]) @ np.abs(w[e]).T
    return out, size


# ----------------------------------------------------------------------------- router training

def balance_loss(probs, idx, coef, valid=None):
    """(loss, counts, gradient per expert of any valid token's probability)."""
    T, M = probs.shape
    keep = range(T) if valid is None else [t for t in range(T) if valid[t]]
    k = idx.shape[1]
    counts, mass = np.zeros(M, np.int64), np.zeros(M)
    for t in keep:
        mass += probs[t]
        for e in idx[t]:
            counts[e] += 1
    n = len(keep)
    if n == 0:
        return 0.0, counts, np.zeros(M)
    f, p = counts / (n * k), mass / n
    return coef * M * float(f @ p), counts, coef * M * f / n


def gate_loss(logits_local, logits_group, groups, sel, renormalize, d_topk_w, d_probs, cand):
    """The linear functional of one token's gate outputs whose gradient the backward pass gives:
    sum d_topk_w topk_w + sum d_probs g, from the logits through the definition of the gate."""
    M = len(logits_local)
    g = np.zeros(M)
    live = [i for i, grp in enumerate(groups) if any(e in cand for e in grp)]
    u = np.array([logits_group[i] for i in live])
    pg = np.exp(u - u.max()) / np.exp(u - u.max()).sum()
    for share, i in zip(pg, live):
        members = [e for e in groups[i] if e in cand]
        l = np.array([logits_local[e] for e in members])
        pl = np.exp(l - l.max()) / np.exp(l - l.max()).sum()
        g[members] = share * pl
    w = g[sel]
    if renormalize:
        w = w / w.sum()
    return float(w @ d_topk_w + g @ d_probs)


def gate_backward(g, idx, groups, renormalize, d_topk_w=None, d_probs=None, d_balance=None, valid=None):
    """Gradients of the local and group logits [T][M], [T][K] by the chain rule with full Jacobians,
    and a bound on the terms each is a sum of (the sums of magnitudes)."""
    T, M = g.shape
    K = len(groups)
    dl, du = np.zeros((T, M)), np.zeros((T, K))
    dl_abs, du_abs = np.zeros((T, M)), np.zeros((T, K))
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        dg, mag = np.zeros(M), np.zeros(M)
        if d_probs is not None:
            dg += d_probs[t]
            mag += np.abs(d_probs[t])
        if d_balance is not None:
            dg += d_balance
            mag += np.abs(d_balance)
        if d_topk_w is not None:
            sel, dw = idx[t], np.asarray(d_topk_w[t], np.float64)
            size = np.abs(dw)
            if renormalize:
                S = g[t, sel].sum()
                w = g[t, sel] / S
                jac = (np.eye(len(sel)) - np.outer(w, np.ones(len(sel)))) / S  # dw_j / dg_l at [l][j] transposed
                size = (size + np.abs(dw) @ w) / S
                dw = jac.T @ dw
            for j, e in enumerate(sel):
                dg[e] += dw[j]
                mag[e] += size[j]
        for k, grp in enumerate(groups):
            P = g[t, grp].sum()
            if P > 0:
                p = g[t, grp] / P
                dl[t, grp] = P * (np.diag(p) - np.outer(p, p)) @ dg[grp]
                dl_abs[t, grp] = P * (np.diag(p) + np.outer(p, p)) @ mag[grp]
        total, total_abs = float(g[t] @ dg), float(g[t] @ mag)
        for k, grp in enumerate(groups):
            du[t, k] = g[t, grp] @ dg[grp] - g[t, grp].sum() * total
            du_abs[t, k] = g[t, grp] @ mag[grp] + g[t, grp].sum() * total_abs
    return dl, du, dl_abs, du_abs
