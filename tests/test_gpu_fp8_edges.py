"""The 8-bit products and expert layers at values and routings where they can go wrong, on the GPU."""
import numpy as np
import pytest
import torch

from paper_2508_06024_amd import ec2moe as E
from tests.gpu_common import say
from tests.test_gpu_fp8 import DEV, up

pytestmark = pytest.mark.gpu


def _experts(rng, M, d, H, rows):
    """8-bit expert weights of about unit gain."""
    return E.fp8_quantize(up(rng.normal(size=(M, rows, d)) * d ** -0.5), 128), E.fp8_quantize(up(rng.normal(size=(M, d, H)) * H ** -0.5), 128)


# ----------------------------------------------------------------------------- values that are not finite

# the first two routings leave float16 rows between the experts and the combine (the second with a split last round), the
# third float32 rows
@pytest.mark.parametrize("T,M,k,d,H", [(4200, 2, 2, 1152, 512), (4300, 2, 2, 2048, 2048), (40, 2, 2, 256, 512)])
@pytest.mark.parametrize("kind", ["nan", "inf"])
def test_columns_beside_one_that_is_not_finite_are_as_without_it(T, M, k, d, H, kind):
    """One row of the output weights makes one output column NaN or infinite; the others, large in one block of 128 and
    small in the next, are what they are with zeros in that row."""
    say(f"fp8_moe_forward beside a column of {kind} T={T} d={d} H={H}")
    rng = np.random.default_rng(T)
    idx = up(np.stack([rng.permutation(M)[:k] for _ in range(T)]), torch.int32)
    w = up(np.full((T, k), 0.5))
    x = up(np.abs(rng.normal(size=(T, d))), torch.bfloat16)
    # columns of magnitude 2^100 in the first block (2^115 beside the infinity), 2^-60 in the second
    (w_in, s_in), (w_dn, s_dn) = _experts(rng, M, d, H, H)
    w_in = w_in.float().abs().to(E.FP8)  # hidden values above zero: sums of one sign below
    s_dn[:, 0] = 2.0 ** 100 if kind == "nan" else 2.0 ** 112
    s_dn[:, 1] = 2.0 ** -60
    w_dn = w_dn.float()
    w_dn[:, :256] *= 2.0 ** -6
    w_dn = w_dn.to(E.FP8)
    bad = [5, 200] if kind == "nan" else [5]
    code = w_dn.view(torch.uint8)
    code[:, bad] = 0
    call = lambda: E.fp8_moe_forward(x, idx, w, w_in, s_in, w_dn, s_dn, activation="relu")
    ref = call()
    assert torch.isfinite(ref).all()
    assert (ref[:, :128].abs().amax(dim=1) > 2.0 ** 90).all() and (ref[:, 128:256].abs().amax(dim=1) < 2.0 ** -30).all()
    assert (ref[:, 128:200] != 0).float().mean() > 0.99  # two experts' rows may cancel
    code[:, bad] = 0x7f if kind == "nan" else 0x7e  # NaN; 448, whose sums pass 2^128
    got = call()
    keep = torch.ones(d, dtype=torch.bool, device=DEV)
    keep[bad] = False
    assert torch.equal(got[:, keep], ref[:, keep])
    assert (torch.isnan(got[:, bad]) if kind == "nan" else got[:, bad] == float("inf")).all()


# ----------------------------------------------------------------------------- sums of products of unequal size

def _cancelling(rng, rows, k, sign, low, high):
    """Rows of e4m3 values whose runs of 8 begin 448, sign 448 and go on with three small whole numbers and zeros: of a row
    of either sign the first two products cancel, and the others lie up to 17 bits below them."""
    v = rng.integers(low, high + 1, size=(rows, k // 8, 8)).astype(np.float64)
    v[:, :, 0], v[:, :, 1] = 448.0, sign * 448.0
    v[:, :, 5:] = 0
    return v.reshape(rows, k)


@pytest.mark.parametrize("act", ["relu", "swiglu"])
@pytest.mark.parametrize("T,M,d,H", [(6, 2, 256, 256), (40, 64, 256, 1024), (600, 2, 256, 256), (9000, 4, 128, 512), (3000, 2, 2048, 1024)])
def test_hidden_rows_of_a_float32_layer_are_sums_of_exact_products(T, M, d, H, act):
    """Rows of scale 1 whose large products cancel: the hidden sums are whole numbers below 2^24, which float32 sums of exact
    products give whatever their order. The output weights are identities (on 256 columns of H), so that the output is the
    quantised hidden row itself."""
    say(f"fp8_moe_forward float32 exact hidden rows T={T} M={M} d={d} H={H} {act}")
    rng = np.random.default_rng(T + H)
    n = min(d, H)
    x = _cancelling(rng, T, d, 1.0, 1, 4)  # blocks' largest value 448: the scale is 1
    rows = E.w_in_rows(H, act)
    w = np.stack([_cancelling(rng, rows, d, -1.0, -3, 4) for _ in range(M)])
    if act == "swiglu":
        w[:, :H] = np.abs(w[:, :H])  # gates of 32 and more: silu(g) = g in float32
        w[:, :H, 1::8] *= -1
    w_dn = np.zeros((M, d, H))
    w_dn[:, np.arange(n), np.arange(n)] = 1.0
    ones = lambda *shape: torch.ones(shape, device=DEV)
    idx = rng.integers(0, M, size=(T, 1)).astype(np.int32)
    h = np.empty((T, rows))
    for e in range(M):
        own = idx[:, 0] == e
        h[own] = x[own] @ w[e].T
    h = np.maximum(h, 0) if act == "relu" else h[:, :H] * h[:, H:]
    assert np.abs(h).max() < 2 ** 24 and (act == "relu" or np.abs(h).min(axis=1).max() > 0)
    y = E.fp8_moe_forward(up(x), up(idx, torch.int32), ones(T, 1), up(w).to(E.FP8), ones(M, rows // 128, d // 128),
                          up(w_dn).to(E.FP8), ones(M, d // 128, H // 128), activation=act)
    q, s = E.fp8_quantize(up(h))
    want = q.float() * s.repeat_interleave(128, dim=1)
    assert torch.equal(y[:, :n], want[:, :n]) and (y[:, n:] == 0).all()


@pytest.mark.parametrize("rows,G,n,k", [(3, 1, 300, 512), (300, 64, 1100, 384), (512, 1, 1024, 512), (4096, 1, 1024, 512),
                                        (3000, 8, 1999, 256)])
def test_float32_products_are_sums_of_exact_products(rows, G, n, k):
    """As above for the product by itself: its sums are whole numbers, and exact."""
    say(f"fp8_matmul float32 exact rows={rows} G={G} n={n} k={k}")
    rng = np.random.default_rng(rows + n)
    a, w = _cancelling(rng, rows, k, 1.0, 1, 15), np.stack([_cancelling(rng, n, k, -1.0, -15, 15) for _ in range(G)])
    seg = (np.arange(G + 1) * rows // G).astype(np.int32)
    got = E.fp8_matmul(up(a).to(E.FP8), torch.ones((rows, k // 128), device=DEV), up(w).to(E.FP8),
                       torch.ones((G, -(-n // 128), k // 128), device=DEV), up(seg, torch.int32), out_dtype=torch.float32)
    want = np.concatenate([a[seg[g]:seg[g + 1]] @ w[g].T for g in range(G)])
    assert torch.equal(got, up(want))


# ----------------------------------------------------------------------------- workspaces

@pytest.mark.parametrize("make", [lambda n: torch.empty(n, dtype=torch.uint8), lambda n: torch.empty((n, 2), dtype=torch.uint8, device=DEV)[:, 0]])
def test_workspaces_on_the_host_or_with_gaps_are_refused(make):
    ws, x = make(1 << 22), torch.zeros((64, 128), device=DEV)
    q, s = E.fp8_quantize(x)
    (wi, si), (wd, sd) = E.fp8_quantize(torch.zeros((2, 256, 128), device=DEV), 128), E.fp8_quantize(torch.zeros((2, 128, 128), device=DEV), 128)
    idx, w = torch.zeros((64, 1), dtype=torch.int32, device=DEV), torch.ones((64, 1), device=DEV)
    probs, gate = torch.full((64, 2), 0.5, device=DEV), torch.zeros((2, 128), device=DEV)
    for call in (lambda: E.fp8_matmul(q, s, wi[0], si[0], ws=ws), lambda: E.fp8_moe_forward(x, idx, w, wi, si, wd, sd, ws=ws),
                 lambda: E.balance_loss(probs, idx, ws=ws), lambda: E.group_gate_backward(x, gate, gate, probs, idx, ws=ws)):
        with pytest.raises(ValueError, match="ws"):
            call()
