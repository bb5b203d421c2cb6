"""The router at logits and sizes where single precision, the choice's shortened keys or the launch can go wrong, against
double precision.

Tolerances, fixed beforehand.  A probability is at most one, and an exponent x that is off by |x| 2^-24 moves it by at most
|x| e^x 2^-24 < 2^-24: weights and probabilities may be off by 32 2^-24 of one, sums of n rows by 64 2^-24 n, gradients
by the same share of the largest factor that they are made of.  Whole numbers have to be equal."""
import subprocess
import sys

import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
import test_gpu_train_ops as ops
import train_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]
ctx = ops.ctx
NINF = float("-inf")

def test_router_gradient_of_many_groups_repeats_itself(ctx):
    """Weights' gradients go through accumulators that one lane of a warp clears and others add to."""
    import torch
    z, mask, opt, desc = ops.router_case(12000, 64, 4, "fp32", group=3, renorm=True)
    o = ops.router_outputs(12000, 64, 4, 4000)
    ctx.router_forward(desc, z, mask, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    dweight = torch.randn(12000, 4, generator=ops.gen(4)).cuda()
    outs = [torch.empty_like(z) for _ in range(8)]
    for out in outs:
        ctx.router_backward(desc, z, o["index"], o["weight"], o["counts"], o["valid"], None, dweight, out)
    ctx.sync()
    want = ref.router_forward(z, mask, 4, **opt)
    dz, size = ref.router_backward(want, 4, 1.0, dweight, **opt)
    ops.close(outs[0], dz, size, "fp32", 64, "dlogits")
    assert all(torch.equal(out, outs[0]) for out in outs)
