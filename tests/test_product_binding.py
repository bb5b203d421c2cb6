"""Linear layers, dropout and the head's cross entropy seen from the host alone: descriptors, types, the generator of the
tests' masks, and what is refused without a GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

import product_ref as ref
from paper_2408_08586_b200 import binding as rb

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
PAIRS = [("rubick_linear_desc", rb.LinearDesc), ("rubick_dropout_desc", rb.DropoutDesc), ("rubick_head_loss_desc", rb.HeadLossDesc)]


def test_descriptors_are_laid_out_as_in_the_header(tmp_path):
    lines = ['printf("%%s size %%zu\\n", "%s", sizeof(%s));' % (c, c) for c, _ in PAIRS]
    lines += ['printf("%%s %s %%zu\\n", "%s", offsetof(%s, %s));' % (f[0], c, c, f[0]) for c, py in PAIRS for f in py._fields_]
    lines += ['printf("RUBICK_ACT %s %%d\\n", RUBICK_ACT_%s);' % (a, a.upper()) for a in rb.ACTIVATIONS]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rubick.h"\nint main(void) { %s return 0; }\n' % " ".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", INCLUDE, "-o", str(exe), str(src)], check=True)
    got = {tuple(l.split()[:2]): int(l.split()[2]) for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()}
    for c, py in PAIRS:
        assert got[c, "size"] == ctypes.sizeof(py)
        for f in py._fields_:
            assert got[c, f[0]] == getattr(py, f[0]).offset, (c, f[0])
    for name, code in rb.ACTIVATIONS.items():
        assert got["RUBICK_ACT", name] == code


def test_builders_fill_the_distances_in():
    d = rb.linear(3, 40, 24, torch.bfloat16, torch.float32, activation="silu", p=0.5)
    assert (d.ld_x, d.ld_w, d.ld_out, d.ld_res, d.ld_pre, d.dtype, d.btype, d.activation, d.flags) == (40, 24, 24, 24, 24, rb.BF16, rb.F32, 4, 0)
    d = rb.linear(3, 40, 24, torch.float16, by_output=True, ld_out=32)
    assert (d.ld_w, d.ld_out, d.ld_res, d.ld_pre, d.btype, d.flags) == (40, 32, 32, 32, rb.F16, rb.WEIGHT_BY_OUTPUT)
    assert rb.head_loss(3, 40, 24, torch.float16).ld_w == 24 and rb.head_loss(3, 40, 24, torch.float16, by_output=True).ld_w == 40
    assert rb.dropout(3, 40, torch.float32, p=0.1, ld=48).ld_res == 48
    with pytest.raises(KeyError):
        rb.linear(3, 40, 24, torch.bfloat16, activation="tanh")
    for build in (lambda t: rb.linear(4, 64, 64, t), lambda t: rb.dropout(4, 64, t, p=0.1), lambda t: rb.head_loss(4, 64, 64, t)):
        with pytest.raises(ValueError):
            build(torch.float64)


@pytest.mark.parametrize("name", [n for n in rb.EXPORTS if n.startswith(("rubick_linear", "rubick_dropout", "rubick_head_loss"))])
def test_a_call_without_a_context_is_refused(name):
    f = getattr(rb.lib(), name)
    assert f(*([None] * len(f.argtypes))) != 0


def test_the_mask_of_the_tests_is_the_published_generator():
    assert ref.philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert ref.philox((ref.MASK,) * 4, (ref.MASK,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    seed = (-(1 << 40) + 12345, (9 << 32) + 77)
    got = ref.keep(seed, 6, 11, 0.3, first_row=2)
    s, o = (v & ((1 << 64) - 1) for v in seed)
    for row in range(6):
        for col in range(11):
            word = ref.philox((col // 4, row + 2, o & ref.MASK, o >> 32), (s & ref.MASK, s >> 32))[col % 4]
            assert bool(got[row, col]) == (word >= int(torch.tensor(0.3, dtype=torch.float32).double() * 2.0 ** 32))
