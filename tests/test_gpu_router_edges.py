"""The router's training operators at sizes where they can go wrong, on the GPU."""
import numpy as np
import pytest
import torch

from paper_2508_06024_amd import ec2moe as E
from tests.gpu_common import say
from tests.test_gpu_router import test_gate_backward_matches_the_oracle as _matches_the_oracle

pytestmark = pytest.mark.gpu

DEV = "cuda"


# ----------------------------------------------------------------------------- balance loss

def test_balance_loss_of_a_batch_longer_than_a_layer_of_it():
    """18 million tokens, with a descriptor of a wide layer."""
    say("balance_loss of 18 million tokens")
    T, M = 18_000_001, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    p = torch.rand((T, M), device=DEV, generator=g)
    idx = (torch.rand((T, 1), device=DEV, generator=g) < 0.3).int()
    desc = E.moe_desc(T, M, 1, 4096, 14336, 1, torch.bfloat16)
    ws = E.workspace(E.balance_loss_workspace_size(desc), DEV)
    loss, d = torch.empty(1, device=DEV), torch.empty(M, device=DEV)
    counts = torch.empty(M, dtype=torch.int32, device=DEV)
    E.balance_loss_into(desc, p, idx, 0.5, loss, counts, d, ws)
    ones = int(idx.sum())
    assert counts.tolist() == [T - ones, ones]
    f = np.array([T - ones, ones]) / T
    mean = p.double().sum(dim=0).cpu().numpy() / T
    # float32 sums of some 400 positive terms (138 rows a thread, then 256 threads), the rest in float64
    assert abs(float(loss) / (0.5 * M * (f * mean).sum()) - 1) <= 512 * 2.0 ** -24
    np.testing.assert_allclose(d.double().cpu().numpy(), 0.5 * M * f / T, rtol=3 * 2.0 ** -24)
    assert all(torch.equal(a, b) for a, b in zip((loss, counts, d), E.balance_loss(p, idx, 0.5)))


@pytest.mark.parametrize("T,M,value", [(2_000_003, 250, 0.1), (1_000_001, 256, 0.7), (9_000_000, 7, 0.013), (300, 8, 0.3)])
def test_balance_loss_of_long_batches_keeps_float32_precision(T, M, value):
    """Equal probabilities, whose float32 sums in a row would drift one way."""
    say(f"balance_loss of equal probabilities T={T} M={M}")
    p = torch.full((T, M), value, device=DEV)
    idx = (torch.arange(T, device=DEV, dtype=torch.int32) % M).reshape(T, 1)
    loss, counts, _ = E.balance_loss(p, idx, 1.0)
    f = np.bincount(np.arange(T) % M, minlength=M) / T
    assert counts.tolist() == np.bincount(np.arange(T) % M, minlength=M).tolist()
    # sums of 8 float32 terms (7 roundings), a chunk's sum and the loss rounded once each; the rest in float64
    assert abs(float(loss) / (M * float(np.float32(value)) * f.sum()) - 1) <= 10 * 2.0 ** -24


# ----------------------------------------------------------------------------- gate backward

@pytest.mark.parametrize("T,d,M,K,k,keep,renorm,terms,pad,dtype", [
    (70, 128, 64, 1, 6, 64, True, "wb", 0.0, torch.float32),       # one group of a whole wave
    (65, 256, 256, 4, 8, 200, False, "wpb", 0.2, torch.bfloat16),  # groups of 64
    (41, 128, 128, 1, 4, 100, True, "wb", 0.0, torch.bfloat16),    # one group of more than 64
    (130, 128, 256, 1, 16, 256, True, "wpb", 0.0, torch.float32),
    (4099, 128, 192, 2, 8, 150, True, "wb", 0.1, torch.bfloat16),  # groups of 96, more than a token a wave
    (50, 128, 100, 4, 3, 80, False, "wb", 0.0, torch.bfloat16),    # groups of 25
])
def test_gate_backward_of_groups_of_any_size(T, d, M, K, k, keep, renorm, terms, pad, dtype):
    _matches_the_oracle(T, d, M, K, k, keep, False, renorm, terms, pad, dtype)
