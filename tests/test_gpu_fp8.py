"""Parity of the 8-bit quantisation and products with the float64 oracle, on the GPU.

Tolerances count roundings: eps(t) / 2 relative for a rounding to type t. A product of two 8-bit
values is exact, a block of 128 is a float32 sum (each addition off by at most 2^-23 of the sum of
magnitudes, if the matrix core truncates), then two scalings and the sum over the blocks."""
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


def quantised(rng, mats, rows, cols, block_rows, std=1.0):
    """8-bit operands made by the oracle, with their numbers in float64."""
    q = np.empty((mats, rows, cols))
    s = np.empty((mats, -(-rows // block_rows), cols // 128), np.float32)
    for i in range(mats):
        q[i], s[i] = OO.fp8_quantize(rng.normal(size=(rows, cols)) * std, block_rows)
    numbers = np.stack([OO.fp8_numbers(q[i], s[i], block_rows) for i in range(mats)])
    return up(q).to(E.FP8), up(s), numbers


def sum_bound(k):
    """Float32 error of a contraction of width k, relative to the sum of magnitudes."""
    return (128 + 4 + k // 128 + 16) * 2.0 ** -23


# ----------------------------------------------------------------------------- quantisation

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mats,rows,cols,block_rows", [
    (1, 1, 128, 1), (1, 3, 128, 1), (1, 129, 1152, 1), (3, 65, 384, 1), (1, 4096, 512, 1),
    (1, 1, 128, 128), (2, 128, 128, 128), (3, 127, 256, 128), (1, 300, 384, 128), (5, 129, 128, 128),
])
def test_quantize_matches_the_oracle(dtype, mats, rows, cols, block_rows):
    say(f"fp8_quantize {mats}x{rows}x{cols} block_rows={block_rows} {dtype}")
    rng = np.random.default_rng(rows * cols + mats)
    x = up(rng.normal(size=(mats, rows, cols)) * np.exp(rng.normal(size=(mats, rows, 1)) * 2), dtype)
    x[:, 0, :128] = 0.0  # a block of zeros (a row of one)
    q, s = E.fp8_quantize(x, block_rows)
    assert q.dtype == E.FP8 and s.dtype == torch.float32
    for i in range(mats):
        rq, rs = OO.fp8_quantize(down(x[i]), block_rows)
        # the scale is one division of exact values
        np.testing.assert_allclose(down(s[i]), rs, rtol=2.0 ** -24, atol=0)
        # the quotient's rounding (2^-23 relative) moves the code only where it is that near a tie;
        # a quotient with a short binary form is exact, so ties themselves agree
        quo = 448.0 * down(x[i]) / OO.spread(OO.block_amax(down(x[i]), block_rows), rows, block_rows)
        _, near = OO.e4m3_step(quo)
        near_tie = (near <= np.abs(quo) * 2.0 ** -23) & (near > 0)
        got = down(q[i])
        assert (got == rq)[~near_tie].all()
        assert near_tie.mean() < 1e-3


def test_quantize_ties_zero_and_extremes():
    x = torch.zeros((8, 128), device=DEV)
    x[0, 0], x[0, 1:4] = 448.0, torch.tensor([17.0, 19.0, -17.0], device=DEV)  # half way: 16|18, 18|20
    x[1, 0] = 2.0 ** -126
    x[2, 0], x[2, 1] = 3e38, 1.5e38
    x[3, 5] = float("nan")
    x[4, 7] = float("-inf")
    x[5, 0], x[5, 1] = 2.0 ** -9 * 448, 2.0 ** -9 * 2.0 ** -9 * 1.5  # below the smallest normal: 1.5 steps
    x[6, 0] = -1e-30
    q, s = E.fp8_quantize(x, 1)
    v, s = down(q), down(s)[:, 0]
    assert v[0, :4].tolist() == [448, 16, 20, -16]
    assert s[1] == 2.0 ** -100 / 448 or abs(s[1] * 448 * 2.0 ** 100 - 1) < 2.0 ** -23
    assert v[1, 0] == OO.e4m3_round(448 * 2.0 ** -26)  # scaled as if the largest were 2^-100
    assert v[2, 0] == 448 and v[2, 1] == 224 and np.isfinite(s[2])
    assert np.isnan(v[3]).all() and np.isnan(s[3]) and np.isnan(v[4]).all() and np.isnan(s[4])
    assert v[5, 1] == 2.0 ** -8
    assert v[6, 0] == OO.e4m3_round(-448 * float(np.float32(1e-30)) * 2.0 ** 100) and (v[7] == 0).all()
    xb = torch.ones((128, 256), device=DEV, dtype=torch.bfloat16)
    xb[77, 200] = float("nan")
    q, s = E.fp8_quantize(xb, 128)
    assert (down(q)[:, :128] == 448).all() and np.isnan(down(q)[:, 128:]).all() and np.isnan(down(s)[0, 1])


# ----------------------------------------------------------------------------- the product

def _seg(rng, rows, G, tail):
    """Ragged segments, every third empty, `tail` rows behind the last."""
    share = rng.random(G) + 0.05
    share[2::3] = 0
    return np.concatenate([[0], np.round(np.cumsum(share / share.sum()) * (rows - tail))]).astype(np.int32)


MATMULS = [
    # rows, G, n, k, tail
    (1, 1, 1, 128, 0), (1, 1, 4096, 512, 0), (2, 1, 17, 256, 0), (16, 1, 128, 128, 0), (17, 1, 130, 384, 0),
    (33, 1, 255, 640, 0), (100, 1, 1000, 1152, 0), (257, 1, 513, 1024, 0), (700, 1, 384, 256, 0),
    (5, 4, 129, 256, 0), (40, 16, 200, 512, 3), (130, 3, 257, 384, 0), (333, 7, 260, 512, 11),
    (1200, 2, 514, 768, 9), (64, 256, 32, 128, 0), (2500, 5, 640, 1280, 1), (1111, 4, 1025, 1024, 30),
    # enough 256 x 256 tiles: whole rounds and less, ragged rows and columns, the last round split along K (an even and an
    # odd number of blocks, a chunk without any), widths that no 16-byte store fits
    (6144, 1, 2176, 384, 0), (5000, 3, 2184, 512, 7), (5000, 3, 2181, 512, 7), (3328, 1, 2304, 2048, 0),
    (2200, 4, 2056, 2176, 100), (8448, 1, 2048, 2176, 0), (16640, 1, 1024, 256, 0), (8448, 1, 2048, 2048, 0),
    (8700, 4, 2056, 4224, 100),
    # 128-row tiles, groups of some hundred rows
    (1024, 1, 4096, 1024, 0), (3000, 8, 1999, 1152, 41), (900, 8, 2048, 640, 0),
]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,G,n,k,tail", MATMULS)
def test_matmul_matches_the_oracle(rows, G, n, k, tail, out_dtype):
    say(f"fp8_matmul rows={rows} G={G} n={n} k={k} tail={tail} {out_dtype}")
    rng = np.random.default_rng(rows * 7 + n)
    a, a_s, na = quantised(rng, 1, rows, k, 1)
    b, b_s, nb = quantised(rng, G, n, k, 128, std=0.02)
    seg = np.array([0, rows], np.int32) if G == 1 else _seg(rng, rows, G, tail)
    out = torch.full((rows, n), 7.0, dtype=out_dtype, device=DEV)
    got = E.fp8_matmul(a[0], a_s[0], b, b_s, None if G == 1 else up(seg, torch.int32), out=out)
    assert got is out
    ref, size = OO.fp8_matmul(na[0], nb, seg, np.full((rows, n), 7.0))
    lim = np.abs(ref) * HALF[out_dtype] + size * sum_bound(k) * 1.01
    lim[seg[-1]:] = 0.0
    err = np.abs(down(out) - ref)
    assert (err <= lim).all(), f"worst excess {(err - lim).max()}, at {np.unravel_index((err - lim).argmax(), err.shape)}"


def test_matmul_gives_the_same_bits_again_and_for_any_group_order():
    rng = np.random.default_rng(5)
    a, a_s, _ = quantised(rng, 1, 300, 512, 1)
    b, b_s, _ = quantised(rng, 2, 260, 512, 128)
    seg = up([0, 170, 300], torch.int32)
    first = E.fp8_matmul(a[0], a_s[0], b, b_s, seg)
    assert torch.equal(first, E.fp8_matmul(a[0], a_s[0], b, b_s, seg))


def test_matmul_carries_nan_to_its_row_and_columns_only():
    rng = np.random.default_rng(6)
    a, a_s, _ = quantised(rng, 1, 40, 256, 1)
    b, b_s, _ = quantised(rng, 1, 300, 256, 128)
    a_s[0, 3, 1] = float("nan")
    b_s[0, 1, 0] = float("nan")
    got = down(E.fp8_matmul(a[0], a_s[0], b, b_s))
    want = np.zeros((40, 300), bool)
    want[3], want[:, 128:256] = True, True
    assert (np.isnan(got) == want).all()


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,G,n,k", [(1, 1, 300, 256), (600, 64, 256, 256), (512, 1, 1024, 512), (2048, 1, 4096, 512),
                                        (4096, 1, 4096, 512)])
def test_matmul_carries_nan_codes(rows, G, n, k, out_dtype):
    """The code 0x7f (and 0xff) is NaN in the rows and the weights, in every kernel; codes next to it are numbers."""
    say(f"fp8_matmul with NaN codes rows={rows} G={G} n={n} k={k} {out_dtype}")
    a = torch.full((rows, k), 0x7e, dtype=torch.uint8, device=DEV)  # 448
    b = torch.full((G, n, k), 0xfe, dtype=torch.uint8, device=DEV)  # -448
    a[rows - 1, k - 1] = 0x7f
    b[G - 1, 17, 3] = 0xff
    seg = torch.arange(G + 1, device=DEV, dtype=torch.int32) * (rows // G)
    seg[G] = rows
    out = E.fp8_matmul(a.view(E.FP8), torch.ones((rows, k // 128), device=DEV), b.view(E.FP8),
                       torch.ones((G, -(-n // 128), k // 128), device=DEV), seg, out_dtype=out_dtype)
    want = torch.zeros((rows, n), dtype=torch.bool, device=DEV)
    want[rows - 1] = True
    want[int(seg[G - 1]):, 17] = True
    assert torch.equal(torch.isnan(out), want)
    assert (out[~want] == torch.tensor(-448.0 * 448.0 * k, dtype=out_dtype, device=DEV)).all()


def test_matmul_captured_with_a_split_round():
    """Replays of a product whose last round is split, between eager calls on the same workspace."""
    rng = np.random.default_rng(16)
    rows, n, k = 8448, 2048, 2048
    b, b_s = E.fp8_quantize(up(rng.normal(size=(1, n, k)) * 0.02), 128)
    xs = [E.fp8_quantize(up(rng.normal(size=(rows, k)))) for _ in range(2)]
    desc = E.fp8_matmul_desc(rows, 1, n, k, torch.bfloat16)
    need = E.fp8_matmul_workspace_size(desc)
    assert need > 0
    ws, out = E.workspace(need, DEV), torch.empty((rows, n), dtype=torch.bfloat16, device=DEV)
    a, a_s = xs[0][0].clone(), xs[0][1].clone()
    call = lambda: E.fp8_matmul_into(desc, a, a_s, None, b, b_s, out, ws)
    refs = [E.fp8_matmul(*x, b[0], b_s[0]) for x in xs]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(4):
        a.copy_(xs[rep % 2][0])
        a_s.copy_(xs[rep % 2][1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, refs[rep % 2]), f"replay {rep}"
        assert torch.equal(E.fp8_matmul(*xs[1 - rep % 2], b[0], b_s[0], ws=ws), refs[1 - rep % 2])


def test_matmul_with_no_rows_and_all_segments_empty():
    rng = np.random.default_rng(7)
    b, b_s, _ = quantised(rng, 3, 40, 128, 128)
    empty = torch.empty((0, 128), dtype=E.FP8, device=DEV)
    assert E.fp8_matmul(empty, torch.empty((0, 1), device=DEV), b, b_s, up([0, 0, 0, 0], torch.int32)).shape == (0, 40)
    a, a_s, _ = quantised(rng, 1, 20, 128, 1)
    out = torch.full((20, 40), 3.0, device=DEV)
    E.fp8_matmul(a[0], a_s[0], b, b_s, up([0, 0, 0, 0], torch.int32), out=out)
    assert (out == 3.0).all()


def test_matmul_weights_beyond_32_bit_offsets():
    """Group strides past 4 GiB: 40 matrices of 128 MiB, only the last one not zero."""
    G, n, k = 40, 8192, 16384
    say("fp8_matmul with 5 GiB of weights")
    b = torch.zeros((G, n, k), dtype=torch.uint8, device=DEV)
    b[G - 1] = 0x38  # 1.0
    b_s = torch.ones((G, n // 128, k // 128), device=DEV)
    a = torch.full((3, k), 0x38, dtype=torch.uint8, device=DEV).view(E.FP8)
    seg = torch.zeros(G + 1, dtype=torch.int32, device=DEV)
    seg[G] = 3
    seg[1:G] = 1  # one row for group 0, two for the last
    got = E.fp8_matmul(a, torch.ones((3, k // 128), device=DEV), b.view(E.FP8), b_s, seg, out_dtype=torch.float32)
    assert (got[0] == 0).all() and (got[1:] == k).all()


# ----------------------------------------------------------------------------- the layer of experts

def _moe_reference(x, idx, w, w_in, w_down, act, dtype):
    """The definition with the hidden rows quantised, and a bound: roundings of the outputs, and for
    every hidden value so near a rounding border that float32 sums may cross it, one step."""
    T, d = x.shape
    H = w_down.shape[2]
    k = idx.shape[1]
    seg, src, inv = O.permute(idx, w_down.shape[0])
    qx = OO.fp8_numbers(*OO.fp8_quantize(x, 1), 1)
    y_perm, lim_perm = np.zeros((T * k, d)), np.zeros((T * k, d))
    for e in range(w_down.shape[0]):
        rows = slice(int(seg[e]), int(seg[e + 1]))
        if seg[e] == seg[e + 1]:
            continue
        xr = qx[src[rows]]
        h, size = xr @ w_in[e].T, np.abs(xr) @ np.abs(w_in[e]).T
        dh = size * sum_bound(d)
        if act == "relu":
            h = np.maximum(h, 0)
        else:
            g, u, dg, du = h[:, :H], h[:, H:], dh[:, :H], dh[:, H:]
            silu = O.silu(g)
            # |silu'| <= 1.1; exponential and reciprocal of the hardware within a few units
            h, dh = silu * u, 1.1 * dg * np.abs(u) + np.abs(silu) * du + 8 * 2.0 ** -23 * np.abs(silu * u)
        amax = OO.spread(OO.block_amax(h, 1), h.shape[0], 1)
        damax = np.repeat(dh.reshape(h.shape[0], -1, 128).max(axis=2), 128, axis=1)
        quo = 448.0 * h / amax
        step, near = OO.e4m3_step(quo)
        cross = near <= 448.0 * (dh + damax * np.abs(h) / amax) / amax + np.abs(quo) * 2.0 ** -23
        q = OO.e4m3_round(quo) * amax / 448.0
        slip = np.where(cross, step, 0.0) * amax / 448.0 + np.abs(q) * (damax / amax + 2.0 ** -23)
        y_perm[rows] = q @ w_down[e].T
        lim_perm[rows] = slip @ np.abs(w_down[e]).T + (np.abs(q) @ np.abs(w_down[e]).T) * sum_bound(H) \
            + np.abs(y_perm[rows]) * HALF[dtype]
    y, lim = np.zeros((T, d)), np.zeros((T, d))
    for t in range(T):
        for j in range(k):
            p = inv[t * k + j]
            y[t] += w[t, j] * y_perm[p]
            lim[t] += w[t, j] * (lim_perm[p] + np.abs(y_perm[p]) * (k + 1) * 2.0 ** -24)
    return y, lim * 1.05 + np.abs(y) * HALF[dtype]


@pytest.mark.parametrize("T,M,k,keep,d,H,act,dtype,skew", [
    (1, 4, 1, 4, 128, 128, "swiglu", torch.bfloat16, 0.0),
    (1, 8, 8, 8, 256, 384, "swiglu", torch.float32, 0.0),
    (7, 8, 2, 6, 384, 256, "relu", torch.bfloat16, 0.0),
    (64, 16, 2, 12, 256, 640, "swiglu", torch.bfloat16, 1.1),
    (33, 64, 6, 20, 128, 128, "swiglu", torch.float32, 0.5),
    (300, 4, 2, 4, 512, 384, "swiglu", torch.bfloat16, 0.0),
    (700, 3, 2, 2, 256, 512, "relu", torch.float32, 0.0),
    (1500, 2, 1, 2, 384, 256, "swiglu", torch.bfloat16, 0.0),
    (1100, 2, 2, 2, 256, 1152, "swiglu", torch.bfloat16, 0.0),
    # hidden rows quantised by the 256 x 256 tiles, and by the sum over their split last round
    (4200, 2, 1, 2, 512, 1152, "swiglu", torch.bfloat16, 0.0),
    (4200, 2, 1, 2, 512, 2432, "relu", torch.bfloat16, 0.5),
    (2600, 2, 1, 2, 2048, 1152, "swiglu", torch.bfloat16, 0.0),
    (2600, 2, 1, 2, 2048, 1152, "swiglu", torch.float32, 0.0),
    (2600, 2, 1, 2, 2176, 2432, "relu", torch.bfloat16, 0.0),
    # output rows as float16 with scales, the last round split
    (4300, 2, 2, 2, 2048, 2048, "swiglu", torch.bfloat16, 0.0),
    # more assignments than one launch permutes
    (9000, 16, 8, 16, 128, 128, "swiglu", torch.bfloat16, 0.0),
    # 64- and 128-row tiles of the hidden rows
    (600, 8, 2, 8, 1024, 768, "swiglu", torch.bfloat16, 0.0),
    (1000, 8, 2, 8, 640, 1024, "relu", torch.bfloat16, 0.3),
])
def test_moe_forward_matches_the_oracle(T, M, k, keep, d, H, act, dtype, skew):
    say(f"fp8_moe_forward T={T} M={M} k={k} d={d} H={H} {act} {dtype}")
    rng = np.random.default_rng(T + H)
    cand = sorted(rng.choice(M, keep, replace=False).tolist())
    idx, w = W.gen_routing(T, M, k, cand, seed=T + M, skew=skew)
    x = up(rng.normal(size=(T, d)), dtype)
    w_in, w_in_s, n_in = quantised(rng, M, E.w_in_rows(H, act), d, 128, std=d ** -0.5)
    w_dn, w_dn_s, n_dn = quantised(rng, M, d, H, 128, std=H ** -0.5)
    topk_w = up(w, torch.float32)
    y = E.fp8_moe_forward(x, up(idx, torch.int32), topk_w, w_in, w_in_s, w_dn, w_dn_s, activation=act)
    ref, lim = _moe_reference(down(x), idx, down(topk_w), n_in, n_dn, act, dtype)
    err = np.abs(down(y) - ref)
    assert (err <= lim).all(), f"worst excess {(err - lim).max()}"
    # the bound says something: mostly roundings of the output type, slips are rare
    assert np.median(lim) <= (0.05 if dtype == torch.bfloat16 else 0.02) * np.abs(ref).max()
    assert torch.equal(y, E.fp8_moe_forward(x, up(idx, torch.int32), topk_w, w_in, w_in_s, w_dn, w_dn_s, activation=act))


def test_moe_forward_is_near_the_layer_in_full_precision():
    """8-bit experts from bfloat16 ones: each of the four quantised operands is off by at most 2^-4
    relative (uniform within: a third of that in the mean), errors of random sign."""
    rng = np.random.default_rng(9)
    T, M, k, d, H = 96, 8, 2, 512, 768
    idx, w = W.gen_routing(T, M, k, list(range(M)), seed=1, skew=0.0)
    x = up(rng.normal(size=(T, d)), torch.bfloat16)
    w_in, w_dn = up(rng.normal(size=(M, 2 * H, d)) * d ** -0.5, torch.bfloat16), up(rng.normal(size=(M, d, H)) * H ** -0.5, torch.bfloat16)
    full = E.moe_forward(x, up(idx, torch.int32), up(w, torch.float32), w_in, w_dn).float()
    got = E.fp8_moe_forward(x, up(idx, torch.int32), up(w, torch.float32), *E.fp8_quantize(w_in, 128), *E.fp8_quantize(w_dn, 128)).float()
    assert float((got - full).norm() / full.norm()) < 2.0 ** -4 * 2  # sqrt(4) operands, each below 2^-4


def test_moe_forward_on_another_stream_and_captured():
    """A side stream's call, and a captured one replayed between eager calls on the same workspace."""
    rng = np.random.default_rng(10)
    T, M, k, d, H = 48, 8, 2, 256, 256
    idx, w = (up(v, t) for v, t in zip(W.gen_routing(T, M, k, list(range(M)), seed=2, skew=0.0), (torch.int32, torch.float32)))
    w_in, w_dn = E.fp8_quantize(up(rng.normal(size=(M, 2 * H, d)) * 0.06), 128), E.fp8_quantize(up(rng.normal(size=(M, d, H)) * 0.06), 128)
    xs = [up(rng.normal(size=(T, d)), torch.bfloat16) for _ in range(2)]
    refs = [E.fp8_moe_forward(x, idx, w, *w_in, *w_dn) for x in xs]
    desc = E.moe_desc(T, M, 1, d, H, k, torch.bfloat16)
    ws = E.workspace(E.fp8_moe_workspace_size(desc), DEV)
    x, y = xs[0].clone(), torch.empty_like(xs[0])
    call = lambda: E.fp8_moe_forward_into(desc, x, idx, w, *w_in, *w_dn, y, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, refs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(5):
        x.copy_(xs[rep % 2])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, refs[rep % 2]), f"replay {rep}"
        assert torch.equal(E.fp8_moe_forward(xs[1 - rep % 2], idx, w, *w_in, *w_dn, ws=ws), refs[1 - rep % 2])


@pytest.mark.parametrize("T,M,k,d,H,dtype", [
    (37, 4, 2, 256, 256, torch.bfloat16),
    (37, 6, 3, 256, 128, torch.float32),
    (60, 20, 10, 128, 128, torch.bfloat16),   # more slots than the unrolled sums
    (4200, 2, 2, 1152, 512, torch.bfloat16),  # output rows as float16 with scales
])
def test_moe_forward_of_slots_without_an_expert(T, M, k, d, H, dtype):
    """Ids outside [0, M) add nothing, whatever their weight: as with a weight of zero. K is below the
    16 blocks from which sums are split, so that a row's bits do not depend on the other rows."""
    say(f"fp8_moe_forward without experts T={T} M={M} k={k}")
    rng = np.random.default_rng(T + k)
    idx = np.stack([rng.permutation(M)[:k] for _ in range(T)]).astype(np.int32)
    w = rng.random((T, k)).astype(np.float32)
    off = rng.random((T, k)) < 0.3
    off[T // 2] = True  # a padding token
    wild = np.where(rng.random((T, k)) < 0.5, -1, M + rng.integers(0, 1000, (T, k)))
    x = up(rng.normal(size=(T, d)), dtype)
    w_in, w_dn = E.fp8_quantize(up(rng.normal(size=(M, 2 * H, d)) * d ** -0.5), 128), E.fp8_quantize(up(rng.normal(size=(M, d, H)) * H ** -0.5), 128)
    got = E.fp8_moe_forward(x, up(np.where(off, wild, idx), torch.int32), up(w), *w_in, *w_dn)
    ref = E.fp8_moe_forward(x, up(idx, torch.int32), up(np.where(off, 0, w)), *w_in, *w_dn)
    assert torch.equal(got, ref) and (got[T // 2] == 0).all() and got.abs().max() > 0
    none = E.fp8_moe_forward(x, up(wild, torch.int32), up(w), *w_in, *w_dn)
    assert (none == 0).all()


def test_moe_forward_of_two_streams_at_once():
    """Calls on two streams, each with its own workspace and output, in flight together."""
    rng = np.random.default_rng(14)
    M, k, d, H = 8, 2, 512, 512
    w_in, w_dn = E.fp8_quantize(up(rng.normal(size=(M, 2 * H, d)) * 0.05), 128), E.fp8_quantize(up(rng.normal(size=(M, d, H)) * 0.05), 128)
    jobs = []
    for i, T in enumerate((64, 3000)):
        idx, w = W.gen_routing(T, M, k, list(range(M)), seed=i, skew=0.5)
        x, idx, w = up(rng.normal(size=(T, d)), torch.bfloat16), up(idx, torch.int32), up(w)
        desc = E.moe_desc(T, M, 1, d, H, k, torch.bfloat16)
        jobs.append((desc, x, idx, w, E.fp8_moe_forward(x, idx, w, *w_in, *w_dn), torch.zeros_like(x),
                     E.workspace(E.fp8_moe_workspace_size(desc), DEV), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(4):
        for desc, x, idx, w, _, y, ws, stream in jobs:
            with torch.cuda.stream(stream):
                E.fp8_moe_forward_into(desc, x, idx, w, *w_in, *w_dn, y, ws)
    torch.cuda.synchronize()
    for _, _, _, _, ref, y, _, _ in jobs:
        assert torch.equal(y, ref)


def test_layer_with_8_bit_experts():
    """Ec2moeLayer: routing, codec and reconstruction as with bfloat16 experts, the experts' output that
    of fp8_moe_forward on them."""
    from paper_2508_06024_amd.layer import Ec2moeLayer
    from tests.gpu_common import up as up_bits, up_f32
    cfg = W.CONFIGS["small"].scaled(n_tokens=256, ffn_hidden=512)
    inp = W.gen_layer(cfg)
    dt = cfg.dtype
    full_w = up_bits(inp.w_gate_up, dt), up_bits(inp.w_down, dt)
    (wi, si), (wd, sd) = (E.fp8_quantize(t, 128) for t in full_w)
    args = [up_bits(inp.x, dt), inp.mask, up_bits(inp.w_global, dt), up_f32(inp.b_global), up_bits(inp.w_local, dt), up_f32(inp.b_local)]
    kw = dict(n_groups=cfg.n_groups, top_k=cfg.top_k)
    codec = [up_bits(inp.u, dt), up_bits(inp.v, dt)]
    full = Ec2moeLayer(*args, *full_w, *codec, **kw)
    low = Ec2moeLayer(*args, wi, wd, *codec, expert_scales=(si, sd), **kw)
    full.step()
    y = low.step()
    for name in ("topk_idx", "topk_w", "z", "x_hat"):
        assert torch.equal(getattr(full, name), getattr(low, name)), name
    assert torch.equal(y, E.fp8_moe_forward(low.x_hat, low.topk_idx, low.topk_w, wi, si, wd, sd))
    with pytest.raises(ValueError):
        Ec2moeLayer(*args, wi, wd, *codec, **kw)
    with pytest.raises(ValueError):
        Ec2moeLayer(*args, *full_w, *codec, expert_scales=(si, sd), **kw)
    with pytest.raises(ValueError):
        Ec2moeLayer(*args, wi, wd, *codec, expert_scales=(si, sd), overlap=True, **kw)


def test_binding_refuses_wrong_operands():
    x = torch.zeros((4, 128), device=DEV)
    q, s = E.fp8_quantize(x)
    b, bs = E.fp8_quantize(torch.zeros((2, 40, 128), device=DEV), 128)
    seg = torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        E.fp8_quantize(x, 64)
    with pytest.raises(ValueError):
        E.fp8_quantize(x.t())
    with pytest.raises(TypeError):
        E.fp8_quantize(x.half())
    with pytest.raises(E.Ec2moeError):
        E.fp8_quantize(torch.zeros((4, 100), device=DEV))
    with pytest.raises(ValueError):
        E.fp8_quantize(x.cpu())
    with pytest.raises(TypeError):
        E.fp8_matmul(x, s, b, bs, seg)
    with pytest.raises(ValueError):
        E.fp8_matmul(q, s.reshape(-1), b, bs, seg)
    with pytest.raises(ValueError):
        E.fp8_matmul(q, s, b, bs[:, :, :0], seg)
    with pytest.raises(E.Ec2moeError):
        E.fp8_matmul(q, s, b, bs)  # two groups need segments
