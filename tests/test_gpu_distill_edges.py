"""Distillation at logits where single precision can go wrong, against double precision: finite mask values over whole
stretches of the vocabulary, rows far from zero, infinite losses.

Tolerances as in test_gpu_train_ops.py, fixed beforehand: 96 2^-24 of the terms' size, with differences of logits exact in
double precision and every exponent below 2^5 where it counts."""
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
import test_gpu_train_ops as ops
import train_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]
ctx = ops.ctx
NINF = float("-inf")
LOWEST = {"bf16": -3.3895313892515355e38, "fp32": -3.4028234663852886e38, "fp16": -65504.0}


def definition(z, index, teacher, temperature, up=None):
    """The reference on rows moved to their maximum (exactly, in double precision), which changes nothing but the log-sum: at
    1e30 even a double has no room for the logarithm of a sum beside the logits."""
    import torch
    z = z.double().cpu()
    top = z.max(1, keepdim=True)[0]
    want = ref.distill(z - top, index, teacher, temperature, up)
    live = (want["s_lse"] > 0).double()
    return {**want, "lse": want["lse"] + live * torch.nan_to_num(top[:, 0]) / temperature, "s_lse": want["s_lse"] + live * torch.nan_to_num(top[:, 0]).abs() / temperature}


def run(ctx, z, index, teacher, desc, up, backward=True):
    """(loss, lse) of forward, (loss, lse, dz) of the step, dz of backward"""
    import torch
    rows = len(z)
    f = lambda: torch.full((rows,), 9.0, device="cuda")  # noqa: E731
    loss, lse, loss2, lse2 = f(), f(), f(), f()
    ctx.distill_forward(desc, z, index, teacher, loss, lse)
    both, back = ops.like(z), ops.like(z)
    ctx.distill_step(desc, z, index, teacher, up, loss2, lse2, both[0])
    if backward:
        ctx.distill_backward(desc, z, index, teacher, lse, up, back[0])
    ctx.sync()
    ops.guarded(both)
    ops.guarded(back)
    return loss, lse, loss2, lse2, both[0], back[0] if backward else None


# rows per call: a cluster a row, clusters that stay with one, two and eight blocks, rows longer than a cluster
SHAPES = [(8, 5000, 1.0), (32, 50257, 1.0), (3, 270001, 2.0), (1500, 3000, 0.5), (700, 20011, 2.0), (170, 128000, 1.0), (110, 140001, 1.0)]


@pytest.mark.parametrize("rows,vocab,temperature", SHAPES)
@pytest.mark.parametrize("dtype,fill", [("bf16", LOWEST["bf16"]), ("fp32", LOWEST["fp32"]), ("fp16", LOWEST["fp16"]), ("bf16", -1e10), ("fp32", -1e30),
                                        ("fp32", -1e7)])
def test_distill_takes_vocabularies_masked_with_a_finite_value(ctx, rows, vocab, temperature, dtype, fill):
    """A closed vocabulary: all but the first thousand or so, or a stretch in the middle, at the type's lowest value or a large
    negative number.  Such places have no probability and no gradient, and the rest is as if they were not there."""
    import torch
    if dtype == "fp32" and rows * vocab > 15_000_000:
        rows = 15_000_000 // vocab
    z, index, teacher, desc = ops.distill_case(rows, vocab, 12, dtype, "fp32", temperature=temperature)
    if rows > 2:
        z[2, 4:7] = 0.5                                     # (no -inf here: losses stay finite)
    z[0::3, 1100:] = fill
    z[1::3, vocab // 4: vocab - vocab // 4] = fill
    index[0::3] %= 1100
    inner = (index[1::3] >= vocab // 4) & (index[1::3] < vocab - vocab // 4)
    index[1::3] = torch.where(inner, index[1::3] - vocab // 4, index[1::3])
    up = (torch.rand(rows, generator=ops.gen(2, rows)) + 0.5).cuda()
    want = definition(z, index, teacher, temperature, up)
    loss, lse, loss2, lse2, both, back = run(ctx, z, index, teacher, desc, up)
    for name, got, t in (("loss", loss, "fp32"), ("lse", lse, "fp32"), ("loss", loss2, "fp32"), ("lse", lse2, "fp32"), ("dz", both, dtype), ("dz", back, dtype)):
        # (q times the lowest value may lie beyond single precision where T^2 q > T)
        fine = want[name].abs() <= torch.finfo(torch.float32).max
        assert torch.equal(torch.isfinite(got.float()).cpu(), fine) and not torch.isnan(got.float()).any(), name
        ops.close(torch.where(fine.cuda(), got, 0), torch.where(fine, want[name], 0.0), want["s_" + name], t, 96, name)


@pytest.mark.parametrize("rows,vocab", [(6, 5000), (4, 50257), (1200, 1003), (2, 270001)])
@pytest.mark.parametrize("dtype,fill", [("bf16", LOWEST["bf16"]), ("fp32", LOWEST["fp32"]), ("fp32", -1e9), ("fp32", 1e30), ("bf16", -1e6), ("fp16", LOWEST["fp16"])])
def test_distill_takes_rows_of_one_far_value(ctx, rows, vocab, dtype, fill):
    """Rows that are all one value, however large, are uniform; so are those whose other half is far below."""
    import torch
    z, index, teacher, desc = ops.distill_case(rows, vocab, 12, dtype, "fp32", temperature=2.0)
    z[0::2] = fill
    z[1::2] = fill
    z[1::2, ::2] = fill / 2 if fill < 0 else fill * 1.5
    index = torch.where((index >= 0) & (index < vocab), index // 2 * 2, index).contiguous()
    want = definition(z, index, teacher, 2.0)
    loss, lse, loss2, lse2, both, _ = run(ctx, z, index, teacher, desc, None, backward=vocab > 262144)
    names = (("loss", loss, "fp32"), ("loss", loss2, "fp32"), ("lse", lse, "fp32"), ("lse", lse2, "fp32"))
    if vocab <= 262144:                                     # (longer rows have their gradient from the rounded log-sum)
        names += (("dz", both, dtype),)
    for name, got, t in names:
        ops.close(got, want[name], want["s_" + name], t, 96, name)


def test_distill_loss_of_a_masked_entry_is_as_large_as_the_mask(ctx):
    """A teacher's entry that the student masks with the lowest value costs q times that value, which has a place in
    single precision where the value times log2(e) has not."""
    import torch
    z = torch.randn(2, 600, generator=ops.gen(9)).cuda()
    z[:, 100:300] = LOWEST["fp32"]
    index = torch.tensor([[5, 150], [6, 7]], dtype=torch.int32, device="cuda")
    teacher = torch.tensor([[1.0, 0.5], [1.0, 0.5]], device="cuda")
    desc = rb.distill(2, 600, 2, torch.float32)
    want = ref.distill(z, index, teacher, 1.0)
    loss, lse, loss2, lse2, both, _ = run(ctx, z, index, teacher, desc, None)
    for got in (loss, loss2):
        assert torch.isfinite(got).all()
        ops.close(got, want["loss"], want["s_loss"], "fp32", 96, "loss")


@pytest.mark.parametrize("rows,vocab", [(5, 5000), (32, 50257), (3, 140001), (900, 3001), (170, 64000)])
@pytest.mark.parametrize("dtype,middle,spread,temperature", [("fp32", 30000.0, 2.0, 1.0), ("fp32", -5000.0, 2.0, 0.5), ("fp16", 2100.0, 4.0, 1.0),
                                                             ("bf16", 1000.0, 12.0, 1.5)])
def test_distill_loss_of_rows_far_from_zero(ctx, rows, vocab, dtype, middle, spread, temperature):
    """A softmax does not change when a row is shifted: neither does the loss's error, whatever the shift's own rounding."""
    import torch
    z, index, teacher, desc = ops.distill_case(rows, vocab, 12, dtype, "fp32", temperature=temperature)
    g = ops.gen(7, rows, vocab)
    z.copy_(torch.randn(rows, vocab, generator=g) * spread + middle)
    want = ref.distill(z, index, teacher, temperature)
    loss, lse, loss2, lse2, both, _ = run(ctx, z, index, teacher, desc, None)
    for name, got, t in (("loss", loss, "fp32"), ("loss", loss2, "fp32"), ("dz", both, dtype)):
        ops.close(got, want[name], want["s_" + name], t, 96, name)


def test_distill_infinite_losses_are_infinite(ctx):
    """Entries on logits of -inf: the loss is +inf, not any other number, in each of the kernels."""
    import torch
    for rows, vocab in ((6, 5000), (9, 50257), (2100, 1003), (3, 270001)):
        z, index, teacher, desc = ops.distill_case(rows, vocab, 6, "bf16", "fp32")
        z[0, 40:60] = NINF
        index[0, 0] = 45
        teacher[0, 0] = 12.0
        want = ref.distill(z, index, teacher, 1.0)
        loss, lse, loss2, lse2, both, back = run(ctx, z, index, teacher, desc, None)
        fine = torch.isfinite(want["loss"])
        assert not fine[0]
        for got in (loss, loss2):
            assert torch.equal(torch.isfinite(got).cpu(), fine)
            assert torch.equal(got.double().cpu()[~fine], want["loss"][~fine])
            ops.close(got[fine.cuda()], want["loss"][fine], want["s_loss"][fine], "fp32", 96, "loss")
        assert torch.isfinite(both.float()).all() and torch.isfinite(back.float()).all()


@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 7, 9])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,pad,shift", [(3000, 0, 0), (3000, 0, 5), (3000, 2, 3), (3, 0, 1)])
def test_distill_rows_shorter_than_a_copy(ctx, rows, pad, shift, vocab, dtype):
    """Rows of a few bytes lie several to a 16-byte unit: units that reach out of the tensor are not only the first and last row's."""
    z, index, teacher, desc = ops.distill_case(rows, vocab, 2, dtype, "fp32", pad=pad, shift=shift)
    want = ref.distill(z, index, teacher, 1.0)
    loss, lse, loss2, lse2, both, back = run(ctx, z, index, teacher, desc, None)
    for name, got, t in (("loss", loss, "fp32"), ("lse", lse, "fp32"), ("loss", loss2, "fp32"), ("lse", lse2, "fp32"), ("dz", both, dtype), ("dz", back, dtype)):
        ops.close(got, want[name], want["s_" + name], t, 96, name)
