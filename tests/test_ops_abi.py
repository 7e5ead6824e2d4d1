"""The layer operators' C ABI on the host: exports, struct layouts, and what is refused before anything is launched."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2508_05370_amd import binding as B
from paper_2508_05370_amd import ops as torch_ops
import ops_abi as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20      # an address that is aligned and never read: every call here is refused, or has nothing to do


def test_exports_every_declared_symbol():
    src = open(os.path.join(ROOT, "include", "hetsim_ops.h")).read()
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(sim_\w+)\s*\(", src, re.M))
    assert names == set(ops.EXPORTS)
    for n in names:
        assert hasattr(ops.lib(), n), n


def test_structs_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"sim_blocks": ops.Blocks, "sim_norm_args": ops.NormArgs, "sim_norm_grad_args": ops.NormGradArgs,
               "sim_adamw_tensor": ops.AdamWTensor, "sim_adamw_args": ops.AdamWArgs}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "hetsim_ops.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append('  printf("%s size %%zu\\n", sizeof(%s));' % (cname, cname))
        for f, _ in py._fields_:
            lines.append('  printf("%s %s %%zu\\n", offsetof(%s, %s));' % (cname, f, cname, f))
    lines += ["  return 0;", "}"]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines) + "\n")
    exe = tmp_path / "probe"
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    got = {tuple(x.split()[:2]): int(x.split()[2]) for x in out if x}
    for cname, py in structs.items():
        assert got[(cname, "size")] == C.sizeof(py), cname
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


def _blocks(rows=4, cols=200, **over):
    b = ops.Blocks(codes=P, ld=ops.padded(cols), scales=P, ld_s=rows, block_rows=1)
    for k, v in over.items():
        setattr(b, k, v)
    return b


BAD_BLOCKS = [dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 2), dict(ld=255), dict(ld=128),
              dict(ld=264), dict(ld_s=3), dict(block_rows=0), dict(block_rows=64), dict(block_rows=128, ld_s=0)]


def _quantize(x=P, dtype=0, rows=4, cols=200, ld=200, q=None, qt=None):
    return ops.lib().sim_op_quantize(x, dtype, rows, cols, ld, C.byref(q or _blocks()), qt and C.byref(qt), None)


@pytest.mark.parametrize("over", BAD_BLOCKS[1:], ids=str)
def test_quantize_refuses_block_forms(over):
    assert _quantize(q=_blocks(**over)) == B.SIM_EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=P + 1), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(cols=-1),
                                dict(ld=199), dict(rows=1 << 31), dict(q=_blocks(codes=None)),
                                dict(qt=_blocks(200, 4, block_rows=128)), dict(qt=_blocks(199, 4)), dict(qt=_blocks(200, 200, ld=112))],
                         ids="-".join)
def test_quantize_refuses(kw):
    assert _quantize(**kw) == B.SIM_EINVAL


def _matmul(a=None, b=None, m=4, n=6, k=200, c=P, dtype=0, ldc=6, ws=None, size=0):
    return ops.lib().sim_op_matmul(C.byref(a or _blocks(4, 200)), C.byref(b or _blocks(6, 200)), m, n, k, c, dtype, ldc, 0, ws, size,
                                   None)


@pytest.mark.parametrize("over", BAD_BLOCKS, ids=str)
def test_matmul_refuses_block_forms(over):
    if over.get("block_rows") != 128:
        assert _matmul(a=_blocks(**over)) == B.SIM_EINVAL
    assert _matmul(b=_blocks(6, 200, **over)) == B.SIM_EINVAL


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=-1), dict(k=-1), dict(m=5), dict(n=7), dict(k=300), dict(k=1 << 31), dict(c=None),
                                dict(c=P + 1), dict(dtype=2, c=P + 2), dict(dtype=3), dict(ldc=5)], ids=str)
def test_matmul_refuses(kw):
    assert _matmul(**kw) == B.SIM_EINVAL


def test_workspaces_are_asked_for():
    """A product that is split over k needs its workspace; nothing is launched without."""
    L = ops.lib()
    m, n, k = 128, 128, 1 << 20
    size = L.sim_op_matmul_workspace(m, n, k)
    assert size > 0
    a, b = _blocks(m, k), _blocks(n, k)
    for ws, s in ((None, size), (P, size - 1), (P + 8, size)):
        assert L.sim_op_matmul(C.byref(a), C.byref(b), m, n, k, P, 0, n, 0, ws, s, None) == B.SIM_EINVAL
    for m in (1, 16, 64):            # few rows as well
        size, a, b = L.sim_op_matmul_workspace(m, 256, 1 << 17), _blocks(m, 1 << 17), _blocks(256, 1 << 17)
        assert size >= 2 * m * 256 * 4
        assert L.sim_op_matmul(C.byref(a), C.byref(b), m, 256, 1 << 17, P, 0, 256, 0, P, size - 1, None) == B.SIM_EINVAL
        assert L.sim_op_linear_workspace(m, 256, 1 << 17) >= size
    size = L.sim_op_linear_workspace(40, 100, 300)
    w = _blocks(100, 300)
    assert size >= 40 * 384
    for ws, s in ((None, size), (P, size - 1), (P + 8, size)):
        assert L.sim_op_linear(P, 0, 300, C.byref(w), 40, 100, 300, P, 100, ws, s, None) == B.SIM_EINVAL
    for bad in ((-1, 100, 300), (40, 0, 300), (1 << 31, 100, 300)):
        assert L.sim_op_linear_workspace(*bad) == 0
    assert L.sim_op_norm_backward_workspace(0, 5, 1) == 0 and L.sim_op_norm_backward_workspace(8, 5, 1 << 62) > 0


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=P + 1), dict(dtype=4), dict(ldx=299), dict(t=-1), dict(y=None), dict(y=P + 1),
                                dict(ldy=99), dict(k=400)], ids="-".join)
def test_linear_refuses(kw):
    a = dict(dict(x=P, dtype=0, ldx=300, t=40, n=100, k=300, y=P, ldy=100), **kw)
    w = _blocks(100, 300)
    assert ops.lib().sim_op_linear(a["x"], a["dtype"], a["ldx"], C.byref(w), a["t"], a["n"], a["k"], a["y"], a["ldy"], P, 1 << 40,
                                   None) == B.SIM_EINVAL


def _norm(**kw):
    a = ops.NormArgs(rows=4, hidden=200, act=0, res=0, post=1, pre=1, alpha=1, beta=1, eps=1e-6, h=P, ld_h=200, y=P, ld_y=200,
                     h_out=P, ld_h_out=200, x=P, ld_x=200, rows_per_gate=4)
    for k, v in kw.items():
        setattr(a, k, v)
    return ops.lib().sim_op_norm(C.byref(a), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(hidden=0), dict(hidden=32769), dict(act=3), dict(res=1), dict(post=3), dict(pre=-1), dict(eps=-1.0),
    dict(eps=float("nan")), dict(h=None), dict(h=P + 1), dict(ld_h=199), dict(ld_y=199), dict(y=P + 1), dict(y=None),
    dict(y=None, post=0, gate=P), dict(gate=P, rows_per_gate=0), dict(gate=P + 1), dict(ld_h_out=199), dict(x=None),
    dict(ld_x=199), dict(xq=C.pointer(_blocks())), dict(x=None, xq=C.pointer(_blocks(ld=128))),
    dict(x=None, xq=C.pointer(_blocks(block_rows=128))), dict(pre=0), dict(pre=0, x=None, pre_stats=P), dict(post=0, post_stats=P),
    dict(post=0, post_weight=P), dict(post_weight=P + 2), dict(pre_bias=P + 1)], ids="-".join)
def test_norm_refuses(kw):
    assert _norm(**kw) == B.SIM_EINVAL


def _norm_grad(size=1 << 40, ws=P, **kw):
    a = ops.NormGradArgs(rows=4, hidden=200, act=0, res=0, post=1, pre=1, alpha=1, beta=1, dh_out=P, ld_dh_out=200, dx=P, ld_dx=200,
                         h=P, ld_h=200, y=P, ld_y=200, rows_per_gate=4, post_stats=P, pre_stats=P, dh=P, ld_dh=200, dy=P, ld_dy=200)
    for k, v in kw.items():
        setattr(a, k, v)
    return ops.lib().sim_op_norm_backward(C.byref(a), ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(hidden=0), dict(hidden=32769), dict(act=3), dict(res=1), dict(post=3), dict(pre=3), dict(dx=None),
    dict(ld_dx=199), dict(h=None), dict(ld_h=199), dict(pre_stats=None), dict(post_stats=None), dict(y=None), dict(ld_y=199),
    dict(y=None, post=0), dict(dgate=P), dict(gate=P, rows_per_gate=0), dict(gate=P + 1), dict(ld_dh=199), dict(ld_dy=199),
    dict(ld_dh_out=199), dict(dh_out=P + 1), dict(dy=P + 1), dict(pre=0, dpre_weight=P), dict(post=0, dpost_bias=P),
    dict(dpre_weight=P + 2), dict(ws=None), dict(ws=P + 4), dict(size=100)], ids=str)
def test_norm_backward_refuses(kw):
    assert _norm_grad(**kw) == B.SIM_EINVAL


def _adamw(tensor=None, n=1, **kw):
    t = ops.AdamWTensor(p=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, copy=P, n=10)
    for k, v in (tensor or {}).items():
        setattr(t, k, v)
    a = ops.AdamWArgs(p_dtype=2, grad_dtype=0, copy_dtype=0, state_bits=8, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return ops.lib().sim_op_adamw(C.byref(t) if n else None, n, C.byref(a), None)


@pytest.mark.parametrize("kw", [
    dict(p_dtype=3), dict(grad_dtype=3), dict(copy_dtype=4), dict(state_bits=16), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
    dict(beta2=float("nan")), dict(eps=-1.0), dict(lr=float("inf")), dict(lr=float("nan")), dict(step=0), dict(grad_scale=P + 2),
    dict(skip=P + 1), dict(n=-1), dict(tensor=dict(p=None)), dict(tensor=dict(p=P + 2)), dict(tensor=dict(grad=None)),
    dict(tensor=dict(grad=P + 1)), dict(tensor=dict(m=None)), dict(tensor=dict(v=None)), dict(tensor=dict(m_scale=None)),
    dict(tensor=dict(v_scale=P + 2)), dict(tensor=dict(copy=None)), dict(tensor=dict(copy=P + 1)), dict(tensor=dict(n=-1)), dict(tensor=dict(first=64)),
    dict(tensor=dict(m=P + 2), state_bits=32)], ids=str)
def test_adamw_refuses(kw):
    assert _adamw(**kw) == B.SIM_EINVAL


def test_nothing_to_do():
    assert _adamw(n=0) == B.SIM_OK
    assert _adamw(tensor=dict(n=0, p=None)) == B.SIM_OK
    assert _norm(rows=0, h=None) == B.SIM_OK
    assert _quantize(rows=0, x=None) == B.SIM_OK
    assert _matmul(m=0) == B.SIM_OK and _matmul(n=0) == B.SIM_OK


def test_tensors_are_refused():
    """The binding's own checks: there is no host path, and types and shapes must fit."""
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        torch_ops.quantize(x)
    with pytest.raises(ValueError, match="type"):
        torch_ops.quantize(x.to(torch.int32))
    with pytest.raises(ValueError, match="contiguous"):
        torch_ops.quantize(x.t())
    with pytest.raises(ValueError, match="overlap"):
        torch_ops.quantize(torch.zeros(1, 8).expand(4, 8))
    with pytest.raises(ValueError, match="matrix"):
        torch_ops.quantize(x[0])
    with pytest.raises(ValueError, match="block_rows"):
        torch_ops.quantize(x, block_rows=64)
    with pytest.raises(ValueError, match="GPU"):
        torch_ops.norm_block(x, x)
    with pytest.raises(ValueError, match="32 bits"):
        torch_ops.norm_block(x.half(), x)
    with pytest.raises(ValueError, match="GPU"):
        torch_ops.adamw([x[0]], [x[1]], [x[2]], [x[3]], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="length"):
        torch_ops.adamw([x[0]], [], [x[2]], [x[3]], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="e4m3"):
        torch_ops.linear(x, x, x)
    torch_ops.adamw([], [], [], [], step=1, lr=1e-3)


def test_recorded_tensors_are_refused():
    """No call leaves a history, so none takes a tensor whose gradient is being recorded (on which device it is does not matter)."""
    x, w = torch.zeros(4, 128), torch.zeros(128)
    leaf, inner = torch.zeros(4, 128, requires_grad=True), torch.zeros(4, 128, requires_grad=True) * 2.0
    codes, scales = torch.zeros(8, 128, dtype=torch_ops.E4M3), torch.zeros(1, 8)
    for bad in (leaf, inner):
        for call in (lambda: torch_ops.quantize(bad), lambda: torch_ops.linear(bad, codes, scales), lambda: torch_ops.norm_block(bad),
                     lambda: torch_ops.norm_block(bad, x), lambda: torch_ops.linear_forward(bad, x),
                     lambda: torch_ops.norm_block_backward(None, x, bad, pre_stats=torch.zeros(2, 4))):
            with pytest.raises(ValueError, match="no_grad"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
                call()
    with pytest.raises(ValueError, match="GPU"):
        torch_ops.quantize(inner.detach())
    # an optimizer step writes to parameters
    with pytest.raises(ValueError, match="GPU"):
        torch_ops.adamw([leaf], [x], [x], [x], step=1, lr=1e-3)


def test_more_columns_than_a_launch_takes():
    """Tiles of one row's worth of columns are not split over launches: refused before any."""
    cols = (1 << 31) - 127
    for block_rows in (1, 128):
        q, qt = _blocks(1, cols, block_rows=block_rows), _blocks(cols, 1, block_rows=block_rows)
        assert _quantize(rows=1, cols=cols, ld=cols, q=q, qt=qt) == B.SIM_EINVAL
    assert _quantize(rows=1, cols=1 << 31, ld=1 << 31, q=_blocks(1, 1 << 31)) == B.SIM_EINVAL
