"""Refusals of the training objectives' entry points on the CPU, and the layouts
of their structures."""
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


@pytest.mark.parametrize("name", ["arc_policy_config", "arc_preference_config"])
def test_layouts_match_the_header(name, tmp_path):
    kind = getattr(_lib, name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "libarctopk.h"\n'
                   f'int main(void){{printf("%zu", sizeof({name}));'
                   + "".join(f'printf(" %zu", offsetof({name}, {f}));' for f, _ in kind._fields_)
                   + 'printf(" %d %d %d %d %d", ARC_POLICY_TOTALS, ARC_PREFERENCE_TOTALS,'
                   ' ARC_PREFERENCE_SIGMOID, ARC_PREFERENCE_HINGE, ARC_PREFERENCE_SQUARED);'
                   ' return 0;}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    vals = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                           check=True).stdout.split()]
    assert vals[0] == ctypes.sizeof(kind)
    assert vals[1:-5] == [getattr(kind, f).offset for f, _ in kind._fields_]
    assert vals[-5:] == [arc.ARC_POLICY_TOTALS, arc.ARC_PREFERENCE_TOTALS,
                         arc.ARC_PREFERENCE_SIGMOID, arc.ARC_PREFERENCE_HINGE,
                         arc.ARC_PREFERENCE_SQUARED]


def test_null_contexts():
    p = arc.arc_policy_config(0.2, 0.2, 0.0, 0.0, 0.0, 1.0)
    q = arc.arc_preference_config(0, 0, 0.1, 0.0, 0.0, 1.0)
    n = [None] * 13
    assert refused(L.arc_tokens_policy(None, ctypes.byref(p), 0, None, 4, *n, 4))
    assert refused(L.arc_tokens_policy_terms(None, ctypes.byref(p), 0, *n))
    assert refused(L.arc_tokens_preference(None, ctypes.byref(q), 0, None, 4, None, 0, *n[:10],
                                           4))
    assert refused(L.arc_tokens_preference_terms(None, ctypes.byref(q), 0, None, None, 0,
                                                 *n[:7]))
