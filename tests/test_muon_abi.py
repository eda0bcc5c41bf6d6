"""Refusals of the matrix optimizer's entry points on the CPU, and the layouts of
its structures: every invalid argument is found before any device work."""
import ctypes
import os
import subprocess

import pytest

import paper_2510_26709_amd as arc
from paper_2510_26709_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = _lib._lib
NAN, INF = float("nan"), float("inf")


def refused(status):
    return status == arc.ARC_ERR_INVALID and arc.arc_last_error() != ""


@pytest.mark.parametrize("name", ["arc_muon_matrix", "arc_muon_config", "arc_muon_step_config"])
def test_layouts_match_the_header(name, tmp_path):
    kind = getattr(_lib, name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "libarctopk.h"\n'
                   f'int main(void){{printf("%zu", sizeof({name}));'
                   + "".join(f'printf(" %zu", offsetof({name}, {f}));' for f, _ in kind._fields_)
                   + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    vals = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                           check=True).stdout.split()]
    assert vals[0] == ctypes.sizeof(kind)
    assert vals[1:] == [getattr(kind, f).offset for f, _ in kind._fields_]


BASE = dict(shapes=[(3, 5), (0, 7), (64, 2)], param_dtypes=[0, 1, 1], grad_dtypes=[1, 0, 0],
            weight_decays=[0.1, 0.0, 0.0], lr_scales=[1.0, 1.0, 0.5])


@pytest.mark.parametrize("override", [
    dict(shapes=[(3, -5), (0, 7), (64, 2)]), dict(shapes=[(2**15 + 1, 2**15 + 1), (0, 7), (4, 2)]),
    dict(shapes=[(1, 2**21 + 1), (0, 7), (4, 2)]), dict(shapes=[(2**14, 2**21), (0, 0), (1, 1)]),
    dict(shapes=[(2**62, 2**62), (0, 0), (1, 1)]), dict(shapes=[(0, 2**22), (1, 1), (1, 1)]),
    dict(param_dtypes=[0, 1, 2]), dict(grad_dtypes=[-1, 0, 0]),
    dict(weight_decays=[0.1, -0.1, 0.0]), dict(weight_decays=[NAN, 0.0, 0.0]),
    dict(lr_scales=[1.0, INF, 1.0]), dict(lr_scales=[NAN, 1.0, 1.0]),
    dict(steps=0), dict(steps=65), dict(steps=-1), dict(reserved=1),
    dict(coefficients=(NAN, 0.0, 0.0)), dict(coefficients=(1.0, INF, 0.0)),
    dict(coefficients=(8.0, 0.0, 0.0)),      # entries beyond the pairs
    dict(coefficients=(3.0, 0.0, 0.0)),      # singular values grow past 2.7
    dict(coefficients=(0.0, 0.0, 7.9)), dict(coefficients=(-1.0, 20.0, -19.0)),
    dict(shapes=[], param_dtypes=[], grad_dtypes=[], weight_decays=[], lr_scales=[])])
def test_create_refuses(override):
    cfg, keep = arc.make_muon_config(**dict(BASE, **override))
    out = ctypes.c_void_p(123)
    assert refused(L.arc_muon_create(ctypes.byref(cfg), None, ctypes.byref(out)))
    assert out.value is None
    del keep


def test_null_contexts_and_arguments():
    ok, keep = arc.make_muon_config(**BASE)
    sc = arc.arc_muon_step_config(0.1, 0.9, 1, 0)
    assert refused(L.arc_muon_create(None, None, ctypes.byref(ctypes.c_void_p())))
    assert refused(L.arc_muon_create(ctypes.byref(ok), None, None))
    ok.matrices = None
    assert refused(L.arc_muon_create(ctypes.byref(ok), None, ctypes.byref(ctypes.c_void_p())))
    assert refused(L.arc_muon_orthogonalize(None, None, None))
    assert refused(L.arc_muon_step(None, ctypes.byref(sc), None, None, None, None, None))
    assert L.arc_muon_state_elems(None) == L.arc_muon_state_offset(None, 0) == -1
    assert L.arc_muon_destroy(None) == arc.ARC_OK
    del keep


def test_coefficients_of_each_step():
    with pytest.raises(ValueError):
        arc.make_muon_config(**BASE, steps=3, coefficients=[(1.5, -0.5, 0.0)] * 2)
    with pytest.raises(ValueError):
        arc.make_muon_config(**BASE, steps=2, coefficients=[(1.5, -0.5), (1.5, -0.5)])
    cfg, keep = arc.make_muon_config(**BASE, steps=2, coefficients=(1.5, -0.5, 0.0))
    assert [cfg.coefficients[k] for k in range(6)] == [1.5, -0.5, 0.0] * 2
    del keep
