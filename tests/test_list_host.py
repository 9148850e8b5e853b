"""CPU: the calls over lists of arrays refuse what they cannot take, before anything reaches a device (no context is given, the
pointers are numbers)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2504_05295_b200 import binding, build

INVALID, SHAPE, ALIGN, ALIAS = -1, -2, -3, -4
BASE = 1 << 40
F32, BF16 = binding.DION_F32, binding.DION_BF16


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def grad(rows=4, cols=8, G=BASE, ldg=None, g=F32, out=None, ldo=None, o=None):
    ldg = cols if ldg is None else ldg
    return binding.DionGrad(rows, cols, G, ldg, g, G if out is None else out, ldg if ldo is None else ldo, g if o is None else o)


def param(rows=4, cols=8, at=0, **kw):
    f = dict(X=BASE, ldx=cols, G=BASE + 0x100000, ldg=cols, g_dtype=F32, M=BASE + 0x200000, ldm=cols, m_dtype=F32,
             V=BASE + 0x300000, ldv=cols, X16=None, ldx16=0, lr_scale=1.0, weight_decay=0.0)
    for k in ("X", "G", "M", "V"):
        f[k] += at
    f.update(kw)
    return binding.DionParam(rows, cols, *f.values())


def rule(beta1=0.9, beta2=0.95, eps=1e-8, step=1, step_dev=None, grad_scale=None):
    return binding.DionRule(beta1, beta2, eps, step, step_dev, grad_scale)


def norm(lib, *grads, count=None, kind=0, max_norm=1.0, norm_out=0x1000, each=None, coef=None, ctx=None):
    arr = (binding.DionGrad * len(grads))(*grads)
    return lib.dion_grad_norm(ctx, arr, len(grads) if count is None else count, kind, max_norm, norm_out, each, coef, None)


def clip(lib, *grads, max_norm=1.0, kind=0, norms=None, num=0, norm_out=None, coef=None):
    arr = (binding.DionGrad * len(grads))(*grads)
    return lib.dion_clip_grads(None, arr, len(grads), max_norm, kind, norms, num, norm_out, coef, None)


def step(lib, *params, r=None, lr=0.1, adamw=True):
    arr = (binding.DionParam * len(params))(*params)
    fn = lib.dion_adamw_step if adamw else lib.dion_lion_step
    return fn(None, arr, len(params), ctypes.byref(rule() if r is None else r), lr, None)


def test_struct_layout_matches_header(tmp_path):
    kinds = {"dion_grad": binding.DionGrad, "dion_param": binding.DionParam, "dion_rule": binding.DionRule}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "dion.h"', 'int main(void) {']
    want = []
    for name, kind in kinds.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(kind))
        for f, _ in kind._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(kind, f).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ['  return 0;', '}']))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", inc, str(src), "-o", str(exe)], check=True)
    assert [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def test_no_context(lib):
    # what is in order reaches the context and finds none
    assert norm(lib, grad()) == INVALID and clip(lib, grad()) == INVALID
    assert step(lib, param()) == INVALID and step(lib, param(), adamw=False) == INVALID


@pytest.mark.parametrize("call", [norm, clip])
def test_gradient_refusals(lib, call):
    assert call(lib, grad(rows=-1)) == SHAPE and call(lib, grad(cols=-1)) == SHAPE
    assert call(lib, grad(ldg=7)) == SHAPE
    assert call(lib, grad(rows=1 << 40, cols=1 << 40)) == SHAPE and call(lib, grad(ldg=1 << 62)) == SHAPE
    assert call(lib, grad(G=BASE + 2)) == ALIGN and call(lib, grad(G=BASE + 1, g=BF16)) == ALIGN
    assert call(lib, grad(G=0)) == INVALID and call(lib, grad(g=2)) == INVALID
    assert call(lib, grad(), kind=2) == INVALID and call(lib, grad(), kind=-1) == INVALID
    # an empty array needs no memory, a bf16 one two-byte alignment
    assert call(lib, grad(rows=0, G=None, ldg=0)) == INVALID and call(lib, grad(G=BASE + 2, g=BF16)) == INVALID


def test_norm_refusals(lib):
    assert norm(lib, count=-1) == INVALID
    assert lib.dion_grad_norm(None, None, 1, 0, 1.0, 0x1000, None, None, None) == INVALID
    assert norm(lib, grad(), norm_out=0x1002) == ALIGN and norm(lib, grad(), each=0x1001) == ALIGN
    # outputs over one another or over a gradient; a gradient may stand in the list twice
    assert norm(lib, grad(), norm_out=0x1000, coef=0x1000) == ALIAS
    assert norm(lib, grad(), grad(), norm_out=0x1004, each=0x1000) == ALIAS
    assert norm(lib, grad(), norm_out=BASE + 4) == ALIAS
    assert norm(lib, grad(), grad()) == INVALID
    assert norm(lib, grad(), coef=0x2000, max_norm=float("nan")) == INVALID


def test_clip_refusals(lib):
    nan = float("nan")
    assert clip(lib, grad(), max_norm=-1.0) == INVALID and clip(lib, grad(), max_norm=nan) == INVALID
    assert clip(lib, grad(), norms=0x1000, num=0) == INVALID and clip(lib, grad(), norms=None, num=1) == INVALID
    assert clip(lib, grad(), norms=0x1000, num=2, norm_out=0x1004) == ALIAS
    # the same gradient twice, two that overlap, a result over another gradient, in place with another type or layout
    assert clip(lib, grad(), grad()) == ALIAS
    assert clip(lib, grad(), grad(G=BASE + 64)) == ALIAS and clip(lib, grad(G=BASE + 64), grad()) == ALIAS
    assert clip(lib, grad(out=BASE + 0x1000), grad(G=BASE + 0x1000, out=BASE + 0x2000)) == ALIAS
    assert clip(lib, grad(o=BF16)) == ALIAS and clip(lib, grad(ldo=16)) == ALIAS
    assert clip(lib, grad(out=BASE + 2)) == ALIGN and clip(lib, grad(o=5)) == INVALID
    # neighbours, and column slices of one matrix, do not overlap; slices that share a column do
    assert clip(lib, grad(), grad(G=BASE + 128)) == INVALID
    a, b = grad(ldg=16), grad(G=BASE + 32, ldg=16)
    assert clip(lib, a, b) == INVALID and clip(lib, b, a) == INVALID
    assert clip(lib, a, grad(G=BASE + 28, ldg=16)) == ALIAS
    assert clip(lib, a, grad(G=BASE + 64 + 36, ldg=16)) == ALIAS      # the last column runs into the next row of the first


@pytest.mark.parametrize("adamw", [True, False])
def test_step_refusals(lib, adamw):
    def s(*params, **kw):
        return step(lib, *params, adamw=adamw, **kw)
    assert s(param(rows=-3)) == SHAPE and s(param(ldx=3)) == SHAPE and s(param(ldm=3)) == SHAPE and s(param(ldg=3)) == SHAPE
    assert s(param(X=BASE + 2)) == ALIGN and s(param(X16=BASE + 0x500001, ldx16=8)) == ALIGN
    assert s(param(X=None)) == INVALID and s(param(g_dtype=9)) == INVALID and s(param(m_dtype=-1)) == INVALID
    assert s(param(lr_scale=float("inf"))) == INVALID and s(param(weight_decay=float("nan"))) == INVALID
    assert s(param(), lr=float("nan")) == INVALID
    for bad in (1.0, -0.1, float("nan")):
        assert s(param(), r=rule(beta1=bad)) == INVALID and s(param(), r=rule(beta2=bad)) == INVALID
    assert s(param(), r=rule(grad_scale=0x1002)) == ALIGN
    assert s(param(), param()) == ALIAS and s(param(), param(at=64)) == ALIAS and s(param(M=BASE)) == ALIAS
    assert s(param(G=BASE)) == ALIAS and s(param(X16=BASE + 0x100000, ldx16=8)) == ALIAS
    assert s(param(), r=rule(grad_scale=BASE)) == ALIAS
    assert s(param(), param(at=128)) == INVALID      # neighbours
    if adamw:
        assert s(param(V=None)) == INVALID and s(param(ldv=2)) == SHAPE and s(param(V=BASE)) == ALIAS
        assert s(param(), r=rule(step=0)) == INVALID and s(param(), r=rule(eps=-1.0)) == INVALID
        assert s(param(), r=rule(step_dev=0x1004)) == ALIGN
    else:
        assert s(param(V=None, ldv=0), param(at=128, V=None, ldv=0)) == INVALID


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, 4)
    with pytest.raises(ValueError, match="CUDA"):
        binding.grad_list([t])
    with pytest.raises(ValueError, match="CUDA"):
        binding.param_list([binding.param_desc(t, t, t)])
    with pytest.raises(ValueError, match="as many"):
        binding.grad_list([t], [])


def test_layout_of_tensors():
    one = torch.zeros(6, 10)
    assert binding._layout([one, one]) == (1, 60, [60, 60])
    assert binding._layout([one[:, :4], torch.zeros(6, 4)]) == (6, 4, [10, 4])
    assert binding._layout([one[:1, :4]]) == (1, 4, [4])
    assert binding._layout([one.view(-1)[::2]]) == (30, 1, [2])
    assert binding._layout([torch.zeros(())]) == (1, 1, [1])
    assert binding._layout([one[:, :0]])[:2] in ((0, 0), (1, 0))
    assert binding._layout([torch.zeros(2, 3, 4)]) == (1, 24, [24])
    with pytest.raises(ValueError):
        binding._layout([one.t()])
    with pytest.raises(ValueError):
        binding._layout([torch.zeros(2, 3, 8)[:, :, :4]])
    with pytest.raises(ValueError):
        binding._layout([one, torch.zeros(60)])
    for kind, want in ((2, 0), (2.0, 0), ("2", 0), ("inf", 1), (float("inf"), 1)):
        assert binding._norm_type(kind) == want
    for kind in (1, "fro", None, 0):
        with pytest.raises(ValueError):
            binding._norm_type(kind)
