"""The operators of a training step seen from the host alone: descriptors, types and what is refused without a GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2408_08586_b200 import binding as rb

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def test_descriptors_are_laid_out_as_in_the_header(tmp_path):
    pairs = [("rubick_block_norm_desc", rb.BlockNormDesc), ("rubick_router_desc", rb.RouterDesc), ("rubick_distill_desc", rb.DistillDesc)]
    lines = ['printf("%%s size %%zu\\n", "%s", sizeof(%s));' % (c, c) for c, _ in pairs]
    lines += ['printf("%%s %s %%zu\\n", "%s", offsetof(%s, %s));' % (f[0], c, c, f[0]) for c, py in pairs for f in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rubick.h"\nint main(void) { %s return 0; }\n' % " ".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", INCLUDE, "-o", str(exe), str(src)], check=True)
    got = {tuple(l.split()[:2]): int(l.split()[2]) for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()}
    for c, py in pairs:
        assert got[c, "size"] == ctypes.sizeof(py)
        for f in py._fields_:
            assert got[c, f[0]] == getattr(py, f[0]).offset, (c, f[0])


def test_types_that_no_operator_has_are_refused_by_the_builders():
    for build in (lambda t: rb.block_norm(4, 64, t), lambda t: rb.router(4, 8, 2, t), lambda t: rb.distill(4, 64, 2, t)):
        build(torch.bfloat16)
        with pytest.raises((KeyError, TypeError, ValueError, rb.RubickError)):
            build(torch.float64)


@pytest.mark.parametrize("name", [n for n in rb.EXPORTS if n.startswith(("rubick_block_norm", "rubick_router", "rubick_distill"))])
def test_a_call_without_a_context_is_refused(name):
    f = getattr(rb.lib(), name)
    assert f(*([None] * len(f.argtypes))) != 0
