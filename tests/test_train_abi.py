"""Refusals of the training operators' entry points on the CPU: every invalid
argument is found before any device work."""
import ctypes
import os
import subprocess

import pytest

import paper_2510_26709_amd as arc
from paper_2510_26709_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = _lib._lib


def refused(status):
    return status == arc.ARC_ERR_INVALID and arc.arc_last_error() != ""


@pytest.mark.parametrize("name", ["arc_tokens_config", "arc_optim_tensor", "arc_optim_config",
                                  "arc_adamw_config"])
def test_layouts_match_the_header(name, tmp_path):
    kind = getattr(_lib, name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "libarctopk.h"\n'
                   f'int main(void){{printf("%zu", sizeof({name}));'
                   + "".join(f'printf(" %zu", offsetof({name}, {f}));' for f, _ in kind._fields_)
                   + 'printf(" %d %d", ARC_STATE_BLOCK, ARC_MAX_TOP); return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    vals = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                           check=True).stdout.split()]
    assert vals[0] == ctypes.sizeof(kind)
    assert vals[1:-2] == [getattr(kind, f).offset for f, _ in kind._fields_]
    assert vals[-2:] == [arc.ARC_STATE_BLOCK, arc.ARC_MAX_TOP]


@pytest.mark.parametrize("override", [
    dict(vocab=0), dict(vocab=-1), dict(vocab=2**31), dict(max_rows=0), dict(max_rows=2**31),
    dict(dtype=2), dict(dtype=-1), dict(top=-1), dict(top=33), dict(top=8, vocab=7),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(reserved=1)])
def test_tokens_create_refuses(override):
    cfg = arc.make_tokens_config(**dict(dict(vocab=100, max_rows=4), **override))
    out = ctypes.c_void_p(123)
    assert refused(L.arc_tokens_create(ctypes.byref(cfg), None, ctypes.byref(out)))
    assert out.value is None


BASE = dict(counts=[10, 0, 300], param_dtypes=[0, 1, 1], grad_dtypes=[1, 0, 0],
            weight_decays=[0.1, 0.0, 0.0], lr_scales=[1.0, 1.0, 0.5])


@pytest.mark.parametrize("override", [
    dict(counts=[10, -1, 3]), dict(counts=[2**41, 2**41, 1]), dict(counts=[2**62, 2**62, 2**62]),
    dict(param_dtypes=[0, 1, 2]), dict(grad_dtypes=[-1, 0, 0]),
    dict(weight_decays=[0.1, -0.1, 0.0]), dict(weight_decays=[float("nan"), 0.0, 0.0]),
    dict(lr_scales=[1.0, float("inf"), 1.0]), dict(lr_scales=[-1.0, 1.0, 1.0]),
    dict(state=2), dict(stochastic=2), dict(reserved=1),
    dict(counts=[], param_dtypes=[], grad_dtypes=[], weight_decays=[], lr_scales=[])])
def test_optim_create_refuses(override):
    cfg, keep = arc.make_optim_config(**dict(BASE, **override))
    out = ctypes.c_void_p(123)
    assert refused(L.arc_optim_create(ctypes.byref(cfg), None, ctypes.byref(out)))
    assert out.value is None
    del keep


def test_null_contexts_and_arguments():
    ok, keep = arc.make_optim_config(**BASE)
    tok = arc.make_tokens_config(vocab=10, max_rows=2)
    assert refused(L.arc_optim_create(None, None, ctypes.byref(ctypes.c_void_p())))
    assert refused(L.arc_optim_create(ctypes.byref(ok), None, None))
    assert refused(L.arc_tokens_create(None, None, ctypes.byref(ctypes.c_void_p())))
    assert refused(L.arc_tokens_create(ctypes.byref(tok), None, None))
    ok.tensors = None
    assert refused(L.arc_optim_create(ctypes.byref(ok), None, ctypes.byref(ctypes.c_void_p())))
    assert refused(L.arc_tokens_score(None, 0, None, 0, None, None, None, None, None, None))
    assert refused(L.arc_tokens_grad(None, 0, None, 0, None, None, None, None, None, None, None,
                                     0))
    assert refused(L.arc_tokens_loss(None, 0, None, 0, None, None, None, None, None, None, None,
                                     None, 0))
    assert refused(L.arc_optim_norm(None, None, 1.0, 1.0, None, None))
    assert refused(L.arc_optim_adamw(None, None, 0, None, None, None, None, None, None, None,
                                     None))
    assert L.arc_optim_state_elems(None) == L.arc_optim_state_offset(None, 0) == -1
    assert L.arc_tokens_destroy(None) == L.arc_optim_destroy(None) == arc.ARC_OK
    del keep
