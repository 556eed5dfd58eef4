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
