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

LOWEST = {"bf16": -3.3895313892515355e38, "fp32": -3.4028234663852886e38, "fp16": -65504.0}


def far_rows(experts, dtype, fill):
    """Six rows about `fill`: all of it, one expert above it, half ordinary, all but one, spread by whole exponents, and ordinary."""
    import torch
    g = ops.gen(experts, dtype, fill)
    z = torch.randn(6, experts, generator=g)
    z[0] = fill
    z[1] = fill
    z[1, experts // 2] = fill / 2 if fill < 0 else fill * 1.5
    z[2, : experts // 2] = fill
    z[3, 1:] = fill
    z[4] = fill * (1 - torch.randint(0, 3, (experts,), generator=g) * 2.0 ** -6)
    return z.to(ops.T(dtype)).cuda()


@pytest.mark.parametrize("experts", [7, 16, 64, 128, 256, 600])
@pytest.mark.parametrize("dtype,fill", [("fp32", -1e9), ("fp32", 1e7), ("fp32", -1e4), ("fp32", 2e38), ("fp32", LOWEST["fp32"]),
                                        ("bf16", -1e9), ("bf16", 1e7), ("bf16", LOWEST["bf16"]), ("fp16", LOWEST["fp16"])])
def test_router_takes_logits_far_from_zero(ctx, dtype, fill, experts):
    """Padding that was filled with a finite mask value instead of being masked: such a row is uniform, not NaN."""
    import torch
    z, k = far_rows(experts, dtype, fill), 3
    opt = dict(group_rows=4, coef=0.3, renorm=False)
    want = ref.router_forward(z, None, k, **opt)
    desc = rb.router(6, experts, k, ops.T(dtype), **opt)
    o = ops.router_outputs(6, experts, k, 2)
    ctx.router_forward(desc, z, None, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    ctx.sync()
    for name in ("index", "counts", "valid"):
        assert torch.equal(o[name].cpu().long(), want[name]), name
    one = torch.ones(1, dtype=torch.float64)
    ops.close(o["weight"], want["weight"], one, "fp32", 32, "weight")
    ops.close(o["prob_sum"], want["prob_sum"], 4 * one, "fp32", 64, "prob_sum")
    loss = torch.tensor([want["loss"]], dtype=torch.float64)
    ops.close(o["loss"], loss, loss.abs(), "fp32", 64, "loss")


@pytest.mark.parametrize("experts", [7, 16, 64, 128, 256, 600])
@pytest.mark.parametrize("dtype,fill", [("fp32", -1e9), ("fp32", 1e11), ("fp32", 2e38), ("fp32", LOWEST["fp32"]),
                                        ("bf16", -1e9), ("bf16", 1e11), ("bf16", LOWEST["bf16"]), ("fp16", LOWEST["fp16"])])
def test_router_gradient_takes_logits_far_from_zero(ctx, dtype, fill, experts):
    import torch
    z, k = far_rows(experts, dtype, fill), 3
    for renorm in (False, True):
        opt = dict(group_rows=4, coef=0.3, renorm=renorm)
        want = ref.router_forward(z, None, k, **opt)
        desc = rb.router(6, experts, k, ops.T(dtype), **opt)
        dweight = torch.randn(6, k, generator=ops.gen(3, experts)).cuda()
        out = ops.like(z)
        ctx.router_backward(desc, z, want["index"].int().cuda(), want["weight"].float().cuda(), want["counts"].int().cuda(), want["valid"].int().cuda(),
                            None, dweight, out[0])
        ctx.sync()
        dz, size = ref.router_backward(want, k, 1.0, dweight, **opt)
        most = dweight.abs().max().double().cpu() + 0.3 * experts * want["counts"].max() / (k * 2 * 2)
        ops.close(out[0], dz, size + most, dtype, 64, "dlogits")
        ops.guarded(out)


@pytest.mark.parametrize("experts", [16, 60, 128, 256, 300, 600, 1024])
@pytest.mark.parametrize("k", [1, 2, 5, 8])
def test_router_settles_ties_at_its_last_place(ctx, experts, k):
    """Single-precision logits a few units in the last place apart, many of them equal: whatever lies behind the k-th place
    in the same run of equal upper bits may still be larger."""
    import torch
    g = ops.gen(experts, k)
    z = torch.ones(60, experts)
    z[0, 2] = 1 + 2.0 ** -20                                # behind an exact tie of the first two
    z[1, experts - 1] = 1 + 2.0 ** -20
    z[2:20] += torch.randint(0, 2, (18, experts), generator=g) * 2.0 ** -23
    z[20:40] += (torch.rand(20, experts, generator=g) < 0.05) * 2.0 ** -22
    z[40:] = -z[40:] - torch.randint(0, 3, (20, experts), generator=g) * 2.0 ** -21
    z[50:, : experts // 2] = 2.0                            # places are taken before the run of near ties begins
    z[50:, k - 1: experts // 2] = 1.0
    z = z.cuda()
    want = ref.router_forward(z, None, k, group_rows=60, coef=0.01, renorm=False)
    o = ops.router_outputs(60, experts, k, 1)
    ctx.router_forward(rb.router(60, experts, k, torch.float32), z, None, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    ctx.sync()
    assert torch.equal(o["index"].cpu().long(), want["index"])
    assert torch.equal(o["counts"].cpu().long(), want["counts"])


SIZES = """
import os, sys
sys.path[:0] = [{tests!r}, os.path.dirname({tests!r})]
import torch
import test_gpu_train_ops as ops
import train_ref as ref
from paper_2408_08586_b200 import binding as rb, workloads
ctx = rb.Context(workloads.ENV, device=0)
# smallest shared memory first: a larger shape's opt-in would serve the smaller ones behind it
for rows, experts, k, group in [(50, 26, 26, 50), (50, 27, 26, 50), (50, 28, 26, 50), (3000, 29, 26, 1), (3000, 32, 26, 1),
                                (40, 396, 2, 40), (40, 397, 2, 40), (40, 398, 2, 40), (3000, 445, 1, 1), (3000, 447, 1, 1), (3000, 448, 1, 1)]:
    z = torch.randn(rows, experts, generator=ops.gen(rows, experts)).cuda()
    o = ops.router_outputs(rows, experts, k, -(-rows // group))
    ctx.router_forward(rb.router(rows, experts, k, torch.float32, group_rows=group), z, None, o["index"], o["weight"], o["counts"], o["prob_sum"],
                       o["valid"], o["loss"])
    ctx.sync()
    want = ref.router_forward(z, None, k, group_rows=group, coef=0.01, renorm=False)
    assert torch.equal(o["index"].cpu().long(), want["index"]), (rows, experts)
    assert torch.equal(o["counts"].cpu().long(), want["counts"]), (rows, experts)
print("all of them ran")
"""


def test_router_sizes_about_the_default_shared_memory():
    """In a process of its own: what a call may use must not depend on the calls before it."""
    import os
    got = subprocess.run([sys.executable, "-c", SIZES.format(tests=os.path.dirname(os.path.abspath(__file__)))], capture_output=True, text=True, timeout=600)
    assert got.returncode == 0 and "all of them ran" in got.stdout, got.stderr[-2000:]


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


@pytest.mark.parametrize("rows,group", [(40000, 1), (70001, 2)])
def test_router_gradient_of_groups_that_are_counted_beforehand(ctx, rows, group):
    import torch
    z, mask, opt, desc = ops.router_case(rows, 8, 2, "bf16", group=group, masked=rows // 3)
    groups = -(-rows // group)
    o = ops.router_outputs(rows, 8, 2, groups)
    ctx.router_forward(desc, z, mask, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    out, dw = ops.like(z), torch.randn(rows, 2, generator=ops.gen(6)).cuda()
    ctx.router_backward(desc, z, o["index"], o["weight"], o["counts"], o["valid"], None, dw, out[0])
    ctx.sync()
    want = ref.router_forward(z, mask, 2, **opt)
    assert torch.equal(o["valid"].cpu().long(), want["valid"])
    loss = torch.tensor([want["loss"]], dtype=torch.float64)
    ops.close(o["loss"], loss, loss.abs(), "fp32", 64, "loss")
    dz, size = ref.router_backward(want, 2, 1.0, dw, **opt)
    ops.close(out[0], dz, size, "bf16", 64, "dlogits")
    ops.guarded(out)
