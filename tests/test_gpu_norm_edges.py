"""Block norm at addresses, widths and group lengths where a launch, a copy or an index can go wrong, against double
precision.  Tolerances as in test_gpu_train_ops.py, fixed beforehand: 64 2^-24 of the terms' size."""
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
import test_gpu_train_ops as ops
import train_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]
ctx = ops.ctx


def gradients(ctx, s, opt, desc, rows, cols, shift=0):
    """The backward pass from what the reference's forward pass gives, weight gradients `shift` floats behind 16 bytes."""
    import torch
    x, _, rstd, _, _ = ref.norm_forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], eps=1e-5, **opt)
    x_out = ops.like(s["x"])[0].copy_(x.to(s["x"].dtype))
    rstd = rstd.float().cuda()
    dx, dy = ops.like(s["x"]), ops.like(s["x"])
    buf = torch.full((2 * cols + 32,), 77.0, device="cuda")
    dwa = buf[shift:shift + cols] if opt["after"] else None
    at = (cols + 8 + 3) // 4 * 4 + shift
    dwb = buf[at:at + cols] if opt["before"] else None
    dg = ops.like(s["gate"]) if s["gate"] is not None else None
    ctx.block_norm_backward(desc, x_out, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], dx[0], dy[0], dwa, dg and dg[0], dwb)
    ctx.sync()
    for out in (dx, dy, dg):
        if out is not None:
            ops.guarded(out)
    keep = torch.ones(len(buf), dtype=torch.bool, device="cuda")
    for w, b in ((dwa, shift), (dwb, at)):
        if w is not None:
            keep[b:b + cols] = False
    assert (buf[keep] == 77.0).all()
    got = dict(dx=dx[0], dy=dy[0], dw_after=dwa, dw_before=dwb, dgate=dg and dg[0])
    want = ref.norm_backward(x_out, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], **opt)
    return {k: v for k, v in got.items() if v is not None}, want


def check(got, want, dtype):
    for name, v in got.items():
        ops.close(v, *want[name], "fp32" if name.startswith("dw") else dtype, 64, name)


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("rows,gate,kw", [(1, "one", {}), (1, "none", {}), (1, "token", {}), (2, "group", dict(group=2)), (2, "one", {}), (2, "token", {}),
                                          (3, "one", {}), (4, "group", dict(group=3)), (5, "group", dict(group=5)), (300, "one", {})])
@pytest.mark.parametrize("cols,dtype", [(768, "bf16"), (64, "fp32"), (8192, "fp16"), (771, "bf16"), (16384, "bf16")])
def test_block_norm_weight_gradients_at_any_address(ctx, rows, gate, kw, cols, dtype, shift):
    """Weight gradients are slices of a flat buffer as often as not: any address that a float may have will do."""
    if rows == 300 and cols > 8192:
        rows = 20
    s, opt, desc = ops.norm_case(rows, cols, dtype, dtype, gate, **kw)
    got, want = gradients(ctx, s, opt, desc, rows, cols, shift)
    check(got, want, dtype)


@pytest.mark.parametrize("rows,cols,dtype,pad", [(300, 5501, "fp32", 0), (300, 5500, "fp32", 1), (9, 5501, "fp32", 0), (700, 8191, "bf16", 2), (1200, 515, "fp16", 0)])
def test_block_norm_first_and_last_ragged_rows(ctx, rows, cols, dtype, pad):
    """The first and the last row of a tensor come to their stage partly by hand, with two stages and with more."""
    import torch
    s, opt, desc = ops.norm_case(rows, cols, dtype, dtype, "token", pad=pad, shift=1)
    first, want = gradients(ctx, s, opt, desc, rows, cols)
    check(first, want, dtype)
    for _ in range(6):
        got, _ = gradients(ctx, s, opt, desc, rows, cols)
        assert all(torch.equal(got[k], first[k]) for k in first)


@pytest.mark.parametrize("cols", [1, 2, 3, 5, 7, 9])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,pad,shift", [(9700, 0, 0), (9700, 0, 5), (9700, 2, 3), (3, 0, 1), (2, 0, 0)])
def test_block_norm_of_rows_shorter_than_a_copy(ctx, rows, pad, shift, cols, dtype):
    """Rows of a few bytes lie several to a 16-byte unit: units that reach out of the tensor are not only the first and last row's."""
    import torch
    s, opt, desc = ops.norm_case(rows, cols, dtype, dtype, "group", group=3, pad=pad, shift=shift)
    x_out, h, rstd = ops.like(s["x"]), ops.like(s["x"]), torch.empty(rows, 2, device="cuda")
    ctx.block_norm_forward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out[0], h[0], rstd)
    ctx.sync()
    want_x, want_h, want_r, size_x, size_h = ref.norm_forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], eps=1e-5, **opt)
    ops.close(x_out[0], want_x, size_x, dtype, 64, "x_out")
    ops.close(h[0], want_h, size_h, dtype, 64, "h")
    ops.guarded(x_out)
    ops.guarded(h)
    got, want = gradients(ctx, s, opt, desc, rows, cols)
    check(got, want, dtype)


@pytest.mark.parametrize("group", [2 ** 63 - 1, 2 ** 62 + 5, 2 ** 33, 3001])
@pytest.mark.parametrize("cols", [768, 515, 16384])
def test_block_norm_groups_longer_than_the_rows(ctx, group, cols):
    """A gate row for any number of rows serves all that there are."""
    import torch
    rows = 3000 if cols < 16384 else 200
    s, opt, desc = ops.norm_case(rows, cols, "bf16", "bf16", "one")
    long = rb.block_norm(rows, cols, torch.bfloat16, eps=1e-5, alpha=0.7, group_rows=group)
    outs = []
    for d in (desc, long):
        x_out, h, rstd = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(rows, 2, device="cuda")
        ctx.block_norm_forward(d, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out, h, rstd)
        got, want = gradients(ctx, s, opt, d, rows, cols)
        check(got, want, "bf16")
        outs.append([x_out, h, rstd, *got.values()])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("cols", [512, 771, 16384])
@pytest.mark.parametrize("before", [False, True])
def test_block_norm_gradient_beside_an_infinite_activation(ctx, cols, before):
    """Without a norm after the block, du = alpha g G does not look at y: an infinite y makes its gate's gradient infinite,
    not its own NaN."""
    import torch
    rows = 6
    s, opt, desc = ops.norm_case(rows, cols, "bf16", "bf16", "token", after=False, before=before)
    y = s["y"].clone()
    y[2, 5], y[3, 7] = float("inf"), float("-inf")
    x_out, rstd = s["x"].clone(), torch.full((rows, 2), 0.5, device="cuda")
    outs = []
    for block in (s["y"], y):
        dx, dy, dg = torch.empty_like(x_out), torch.empty_like(x_out), torch.empty_like(s["gate"])
        dwb = torch.empty(cols, device="cuda") if before else None
        ctx.block_norm_backward(desc, x_out if before else None, block, None, s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], dx, dy, None, dg, dwb)
        ctx.sync()
        outs.append((dx, dy, dg))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    off = ~torch.isfinite(outs[1][2].float())
    assert off.sum() == 2 and off[2, 5] and off[3, 7]
