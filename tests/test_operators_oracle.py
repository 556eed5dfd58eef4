"""Pins of the oracle of the 8-bit products and the router's training operators (CPU): the code
table against torch's float8 type, rounding against a search over every code, and the gate's
gradients against central differences of the gate's definition."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO


def test_e4m3_table_is_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(got, OO.e4m3_values())


def test_e4m3_rounding_picks_the_nearest_code():
    rng = np.random.default_rng(0)
    table = OO.e4m3_values()
    table = table[np.isfinite(table)]
    v = np.concatenate([rng.uniform(-500, 500, 400), rng.normal(0, 0.02, 400), table,
                        (table[1:] + table[:-1]) / 2])
    r = OO.e4m3_round(v)
    best = np.abs(v[:, None] - table[None]).min(axis=1)
    np.testing.assert_array_equal(np.abs(v - r), best)
    f = torch.tensor(np.clip(v, -448, 448)).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(r, f)  # ties included


def test_quantised_blocks_are_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(200, 256)) * np.exp(rng.normal(size=(200, 1)) * 3)
    for br in (1, 128):
        q, s = OO.fp8_quantize(x, br)
        assert s.shape == (-(-200 // br), 2) and np.abs(q).max() == 448.0
        err = np.abs(OO.fp8_numbers(q, s, br) - x)
        lim = np.maximum(np.abs(x) * 2.0 ** -4, OO.spread(s, 200, br) * 2.0 ** -10)
        assert (err <= lim * (1 + 1e-12)).all()


@pytest.mark.parametrize("renormalize", [True, False])
def test_gate_gradients_are_the_central_differences(renormalize):
    rng = np.random.default_rng(2)
    M, groups, cand = 9, [[0, 1, 2, 3], [4], [5, 6, 7], [8]], {0, 1, 3, 4, 6, 7}
    for _ in range(5):
        l, u = rng.normal(size=M), rng.normal(size=4)
        sel = np.array([3, 6, 0])
        dw, dp = rng.normal(size=3), rng.normal(size=M)
        # probabilities from the functional itself: its value for unit d_probs
        g = np.array([OO.gate_loss(l, u, groups, sel, False, np.zeros(3), np.eye(M)[e], cand) for e in range(M)])
        assert abs(g.sum() - 1) < 1e-12 and g[8] == 0
        dl, du, _, _ = OO.gate_backward(g[None], sel[None], groups, renormalize, dw[None], dp[None])
        f = lambda l, u: OO.gate_loss(l, u, groups, sel, renormalize, dw, dp, cand)
        h = 1e-5
        for i in range(M):
            e = np.eye(M)[i] * h
            assert abs((f(l + e, u) - f(l - e, u)) / (2 * h) - dl[0, i]) < 1e-8
        for i in range(4):
            e = np.eye(4)[i] * h
            assert abs((f(l, u + e) - f(l, u - e)) / (2 * h) - du[0, i]) < 1e-8


def test_balance_gradient_is_the_difference_of_the_loss():
    rng = np.random.default_rng(3)
    p = rng.dirichlet(np.ones(6), size=10)
    idx = np.argsort(-p, axis=1)[:, :2]
    valid = rng.random(10) < 0.7
    loss, counts, d = OO.balance_loss(p, idx, 0.3, valid)
    assert counts.sum() == 2 * valid.sum()
    for t in range(10):
        for i in range(6):
            q = p.copy()
            q[t, i] += 1e-6
            diff = (OO.balance_loss(q, idx, 0.3, valid)[0] - loss) / 1e-6
            assert abs(diff - (d[i] if valid[t] else 0.0)) < 1e-8
    uniform = np.full((12, 6), 1 / 6)
    idx = np.arange(24).reshape(12, 2) % 6
    assert abs(OO.balance_loss(uniform, idx, 1.0)[0] - 1.0) < 1e-12  # balanced: the coefficient itself
