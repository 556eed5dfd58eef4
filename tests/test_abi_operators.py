"""Refusals of the 8-bit and router entry points, on the host before any HIP call (CPU)."""
import ctypes

import pytest

from paper_2508_06024_amd import ec2moe as E

OK, INVALID, UNSUPPORTED, WS_SMALL = 0, 1, 2, 4
P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 4)


def _quant(x=P, dt=E.BF16, mats=1, rows=4, cols=128, br=1, q=P, s=P):
    return E._lib.ec2moe_fp8_quantize(x, dt, mats, rows, cols, br, q, s, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=7), INVALID), (dict(rows=-1), INVALID), (dict(mats=-1), INVALID), (dict(cols=0), INVALID),
    (dict(br=2), INVALID), (dict(br=0), INVALID), (dict(cols=192), UNSUPPORTED), (dict(x=None), INVALID),
    (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(x=ODD), INVALID), (dict(q=ODD), INVALID), (dict(s=ODD), INVALID),
    (dict(mats=2 ** 31 - 1, rows=2 ** 31 - 1), UNSUPPORTED), (dict(mats=4096, rows=2 ** 20, br=128), UNSUPPORTED),
    (dict(rows=0, x=None, q=None, s=None), OK), (dict(mats=0, x=None, q=None, s=None), OK),
])
def test_quantize(kw, status):
    assert _quant(**kw) == status, E.last_error()


def _mm(rows=4, G=1, n=8, k=128, dt=E.BF16, a=P, a_s=P, seg=None, b=P, b_s=P, out=P):
    d = E.Fp8MatmulDesc(rows, G, n, k, dt)
    return E._lib.ec2moe_fp8_matmul(ctypes.byref(d), a, a_s, seg, b, b_s, out, P, 1 << 40, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=3), INVALID), (dict(rows=-1), INVALID), (dict(G=0), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID),
    (dict(G=257, seg=P), UNSUPPORTED), (dict(k=64), UNSUPPORTED), (dict(n=1 << 20, k=4096), UNSUPPORTED),
    (dict(rows=2 ** 31 - 1, n=1 << 20), UNSUPPORTED), (dict(G=2), INVALID),
    (dict(a=None), INVALID), (dict(a_s=None), INVALID), (dict(b=None), INVALID), (dict(b_s=None), INVALID),
    (dict(out=None), INVALID), (dict(a=ODD), INVALID), (dict(b=ODD), INVALID), (dict(out=ODD), INVALID),
    (dict(rows=0, a=None, b=None, out=None), OK),
])
def test_matmul(kw, status):
    assert _mm(**kw) == status, E.last_error()


def test_matmul_sizes_one_launch_can_hold():
    """Fewer than 2^32 threads over the tiles, 32-bit offsets within a tile: refused beyond, not at, the largest."""
    ok = lambda rows, n, k: E._lib.ec2moe_fp8_matmul_workspace_size(ctypes.byref(E.Fp8MatmulDesc(rows, 1, n, k, E.BF16)),
                                                                    ctypes.byref(ctypes.c_size_t(0)))
    assert ok(2 ** 18, 2 ** 16, 4096) == OK and ok(2 ** 20, 2 ** 14, 128) == OK
    assert ok(2 ** 19, 2 ** 17, 4096) == UNSUPPORTED and ok(2 ** 31 - 1, 2 ** 10, 128) == UNSUPPORTED
    assert ok(1, 1, 2 ** 24 - 128) == OK and ok(1, 1, 2 ** 24) == UNSUPPORTED
    assert ok(2 ** 31 - 1, 1, 2 ** 23) == UNSUPPORTED  # 2^54 bytes of rows: the few-row kernel's tiles


def _desc(**kw):
    base = dict(n_tokens=64, n_experts=8, n_groups=2, d_model=128, ffn_hidden=256, top_k=2, dtype=E.BF16, renormalize=True)
    base.update(kw)
    return E.moe_desc(**base)


def test_matmul_descriptor_and_workspace():
    assert E._lib.ec2moe_fp8_matmul(None, P, P, None, P, P, P, P, 0, None) == INVALID
    n = ctypes.c_size_t(0)
    d = E.Fp8MatmulDesc(4, 1, 8, 128, E.BF16)
    assert E._lib.ec2moe_fp8_matmul_workspace_size(ctypes.byref(d), None) == INVALID
    assert E._lib.ec2moe_fp8_matmul_workspace_size(ctypes.byref(d), ctypes.byref(n)) == OK
    if n.value:
        assert E._lib.ec2moe_fp8_matmul(ctypes.byref(d), P, P, None, P, P, P, P, n.value - 1, None) == WS_SMALL
    assert E._lib.ec2moe_fp8_matmul(ctypes.byref(d), P, P, None, P, P, P, ODD, 1 << 40, None) == INVALID


def test_moe_forward():
    d = _desc()
    need = E.fp8_moe_workspace_size(d)
    call = lambda desc=d, x=P, ws=P, n=need: E._lib.ec2moe_fp8_moe_forward(ctypes.byref(desc), x, P, P, P, P, P, P, P, ws, n, None)
    assert need > 0
    assert call(n=need - 1) == WS_SMALL and call(ws=None) == INVALID and call(x=None) == INVALID and call(x=ODD) == INVALID
    assert call(desc=_desc(d_model=192)) == UNSUPPORTED and call(desc=_desc(top_k=9)) == INVALID
    empty = _desc(n_tokens=0)
    assert call(desc=empty, x=None, n=E.fp8_moe_workspace_size(empty)) == OK


def test_balance_loss():
    d = _desc(n_tokens=100000)
    need = E.balance_loss_workspace_size(d)
    call = lambda probs=P, idx=P, loss=P, ws=P, n=need, desc=d: E._lib.ec2moe_balance_loss(
        ctypes.byref(desc), probs, idx, None, 1.0, None, loss, None, ws, n, None)
    assert need > 0
    assert call(n=need - 1) == WS_SMALL and call(ws=None) == INVALID
    assert call(probs=None) == INVALID and call(idx=None) == INVALID and call(loss=None) == INVALID and call(probs=ODD) == INVALID
    assert call(desc=_desc(n_tokens=-1)) == INVALID


def test_gate_backward():
    d = _desc()
    need = E.gate_backward_workspace_size(d)
    grads = E.GateGrads(1 << 20, None, None, None)

    def call(desc=d, opts=None, g=grads, x=P, wg=P, wl=P, probs=P, idx=P, dx=P, dwg=P, dwl=P, ws=P, n=need):
        return E._lib.ec2moe_group_gate_backward(ctypes.byref(desc), ctypes.byref(opts) if opts else None,
                                                 ctypes.byref(g) if g else None, x, wg, wl, probs, idx, dx, dwg, None, dwl,
                                                 None, ws, n, None)

    assert call(n=need - 1) == WS_SMALL and call(ws=None) == INVALID and call(g=None) == INVALID
    assert call(dwg=None) == INVALID and call(dwl=None) == INVALID
    assert call(x=None) == INVALID and call(wl=None) == INVALID and call(probs=None) == INVALID and call(idx=None) == INVALID
    assert call(dx=ODD) == INVALID and call(dwl=ODD) == INVALID and call(x=ODD) == INVALID
    assert call(opts=E.gate_opts(1)) == UNSUPPORTED and "top_groups" in E.last_error()
    assert call(opts=E.gate_opts(-1)) == INVALID
    assert call(opts=E.gate_opts(0, [3, 4])) == INVALID and call(opts=E.gate_opts(0, [3, 6])) == INVALID
    assert call(desc=_desc(n_groups=3)) == INVALID


def test_descriptor_layouts_are_the_headers(tmp_path):
    """Field offsets of the new structs as a C compiler lays out the header."""
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"ec2moe_fp8_matmul_desc": E.Fp8MatmulDesc, "ec2moe_gate_grads": E.GateGrads}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "ec2moe.h"', "int main(void) {"]
    for s, py in structs.items():
        for f, _ in py._fields_:
            lines.append(f'printf("{s} {f} %zu\\n", offsetof({s}, {f}));')
        lines.append(f'printf("{s} sizeof %zu\\n", sizeof({s}));')
    src, exe = tmp_path / "o.c", tmp_path / "o"
    src.write_text("\n".join(lines + ["return 0;", "}"]) + "\n")
    subprocess.run([cc, "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(root, "include"), str(src),
                    "-o", str(exe)], check=True, capture_output=True)
    got = {tuple(ln.split()[:2]): int(ln.split()[2]) for ln in
           subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()}
    for s, py in structs.items():
        assert got[(s, "sizeof")] == ctypes.sizeof(py)
        for f, _ in py._fields_:
            assert got[(s, f)] == getattr(py, f).offset
