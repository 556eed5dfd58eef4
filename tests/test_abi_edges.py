"""Sizes at which the 8-bit and router entry points decide on the host, before any HIP call (CPU)."""
import ctypes

import pytest

from paper_2508_06024_amd import ec2moe as E

OK, INVALID, UNSUPPORTED = 0, 1, 2


def _balance_size(**kw):
    base = dict(n_tokens=64, n_experts=8, n_groups=2, d_model=128, ffn_hidden=256, top_k=2, dtype=E.BF16)
    desc = E.moe_desc(**{**base, **kw})
    return E._lib.ec2moe_balance_loss_workspace_size(ctypes.byref(desc), ctypes.byref(ctypes.c_size_t(0)))


@pytest.mark.parametrize("kw,status", [
    # the widths of the layer, in its own descriptor or left out, have no part in the loss
    (dict(n_tokens=1 << 20, d_model=4096, ffn_hidden=14336), OK), (dict(d_model=0, ffn_hidden=0), OK),
    (dict(d_model=100, ffn_hidden=-1), OK), (dict(d_model=1 << 20, ffn_hidden=1 << 20), OK),
    # counts are 32-bit numbers
    (dict(n_tokens=2 ** 31 - 1, top_k=1), OK), (dict(n_tokens=2 ** 30, top_k=2), UNSUPPORTED),
    (dict(n_tokens=2 ** 31 - 1, top_k=8), UNSUPPORTED),
    # the routing's own sizes are checked as ever
    (dict(n_experts=0), INVALID), (dict(n_groups=9), INVALID), (dict(top_k=9), INVALID), (dict(n_experts=257), UNSUPPORTED),
    (dict(n_experts=32, top_k=17), UNSUPPORTED), (dict(n_tokens=-1), INVALID), (dict(dtype=5), INVALID),
])
def test_balance_loss_does_not_use_the_layer_widths(kw, status):
    assert _balance_size(**kw) == status, E.last_error()


@pytest.mark.parametrize("sizes", [[8], [3, 3, 2], [1] * 8, []])
def test_group_sizes_of_another_number_of_groups_are_refused(sizes):
    """The library reads one size for each group of the descriptor."""
    import torch
    desc = E.moe_desc(4, 8, 2, 128, 128, 2, E.BF16)
    t = torch.zeros(16)
    opts = E.gate_opts(0, sizes)
    with pytest.raises(ValueError, match="group_sizes"):
        E.group_gate_backward_into(desc, opts, t, t, t, t, t, t)
    with pytest.raises(ValueError, match="group_sizes"):
        E.group_gate_ex(desc, opts, [0xff], t, t, None, t, None, t, t)


def test_moe_desc_refuses_sizes_beyond_32_bits():
    """A field of the descriptor is an int32: more tokens would be taken as their remainder."""
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 64, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            E.moe_desc(n, 8, 2, 128, 256, 2, E.BF16)
    assert E.moe_desc(2 ** 31 - 1, 8, 2, 128, 256, 2, E.BF16).n_tokens == 2 ** 31 - 1


@pytest.mark.parametrize("rows,block_rows,status", [
    (2 ** 31 - 1, 128, UNSUPPORTED), (2 ** 31 - 128, 128, UNSUPPORTED), (2 ** 31 - 1, 1, UNSUPPORTED),
    (2 ** 31 - 1, 2, INVALID),
])
def test_quantize_refuses_more_rows_than_a_launch_takes(rows, block_rows, status):
    p = ctypes.c_void_p(1 << 20)
    assert E._lib.ec2moe_fp8_quantize(p, E.BF16, 1, rows, 128, block_rows, p, p, None) == status, E.last_error()
