"""The training-step operators (block norm, router with balance loss, distillation) against double precision.

Tolerances, fixed beforehand.  A result of type T may be off by its rounding, u |want| with u = 2^-8 (bf16), 2^-11
(fp16, and 2^-24 where it is subnormal), 2^-23 (fp32), plus C 2^-24 times the size of the terms it was summed from.
  block norm   C = 64: a thread adds up to 32 terms, five levels of a warp and five of a block follow, and each term
               carries a handful of roundings of its own.
  router       C = 32: exponentials of a hardware approximation (2 ulp) of an argument below 2^4 (rounded: 2^4 ulp).
  distill      C = 96: the same with arguments below 2^5, over two softmaxes.
Whole numbers have to be equal."""
import zlib

import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
from paper_2408_08586_b200 import workloads
import train_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]

NINF = float("-inf")
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -23}


def T(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


@pytest.fixture(scope="module")
def ctx():
    return rb.Context(workloads.ENV, device=0)


def close(got, want, size, dtype, C, what):
    import torch
    got, want = got.detach().double().cpu().reshape(want.shape), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]) or (torch.isnan(got[~fine]) == torch.isnan(want[~fine])).all(), what
    bound = U[dtype] * want.abs() + C * 2.0 ** -24 * size.double() + (2.0 ** -24 if dtype == "fp16" else 1e-37)
    off = ((got - want).abs() / bound)[fine]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} of the tolerance"


def rows_tensor(g, rows, cols, dtype, pad=0, shift=0, scale=1.0):
    """[rows, cols] cut from a buffer of NaN, `shift` elements behind a 16-byte boundary, rows cols + pad apart."""
    import torch
    buf = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=T(dtype), device="cuda")
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=g) * scale)
    return v


def like(v):
    """A tensor laid out as v, and its buffer with the guard values around the rows."""
    import torch
    rows, cols = v.shape
    ld, shift = v.stride(0) if rows > 1 else max(v.stride(0), cols), v.storage_offset()
    buf = torch.full((shift + rows * ld + 16,), 77.0, dtype=v.dtype, device="cuda")
    return torch.as_strided(buf, (rows, cols), (ld, 1), shift), buf


def guarded(out):
    """Nothing beside the rows was written."""
    import torch
    v, buf = out
    keep = torch.ones(buf.shape, dtype=torch.bool, device="cuda")
    torch.as_strided(keep, v.shape, (v.stride(0), 1), v.storage_offset())[:] = False
    assert (buf[keep] == 77.0).all()


def gen(*key):
    import torch
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


# ------------------------------------------------------------------------------------------------------ block norm

NORM_CASES = [
    # rows, cols, dtype, wtype, gate, keyword options
    (1, 1, "fp32", "fp32", "one", {}),
    (1, 4096, "bf16", "bf16", "one", {}),
    (5, 7, "bf16", "fp32", "token", dict(tanh=True)),
    (33, 64, "fp16", "fp16", "one", dict(offset=True)),
    (130, 96, "bf16", "bf16", "group", dict(group=7)),
    (64, 257, "fp32", "fp32", "group", dict(group=64, pad=3, tanh=True)),
    (200, 768, "bf16", "bf16", "group", dict(group=50)),
    (77, 1280, "fp16", "fp32", "token", dict(tanh=True)),
    (300, 1537, "fp32", "fp32", "none", dict(pad=3)),
    (60, 1537, "bf16", "bf16", "one", dict(pad=1)),
    (37, 2048, "bf16", "bf16", "one", dict(shift=1)),
    (3000, 130, "bf16", "bf16", "group", dict(group=1000)),
    (2500, 40, "fp32", "fp32", "group", dict(group=3)),
    (9, 5120, "bf16", "fp32", "group", dict(group=4, tanh=True, offset=True)),
    (6, 8192, "bf16", "bf16", "one", {}),
    (5, 8200, "fp32", "fp32", "one", {}),
    (4, 16384, "bf16", "bf16", "group", dict(group=2)),
    (3, 16383, "fp16", "fp16", "one", {}),
    (2, 16384, "fp32", "fp32", "none", {}),
    (50, 512, "bf16", "bf16", "none", dict(after=False)),
    (50, 513, "bf16", "bf16", "one", dict(after=False)),
    (50, 512, "fp16", "fp16", "one", dict(before=False)),
    (50, 640, "bf16", "bf16", "none", dict(block=False)),
    (700, 1024, "bf16", "bf16", "one", dict(after=False, before=False)),
    (20, 384, "bf16", "bf16", "one", dict(weights=False)),
    # enough rows for the ring of stages in the forward pass too
    (9700, 64, "bf16", "bf16", "group", dict(group=1000)),
    (9700, 72, "fp32", "fp32", "token", dict(tanh=True)),
    (9700, 128, "fp16", "fp32", "group", dict(group=3, offset=True)),
    (5000, 768, "bf16", "bf16", "one", dict(after=False)),
    (5000, 520, "bf16", "bf16", "group", dict(group=7, before=False)),
    (5000, 512, "bf16", "bf16", "none", dict(after=False, before=False)),
    (5000, 640, "fp32", "fp32", "none", dict(block=False, pad=4)),
    (2400, 2048, "bf16", "fp32", "group", dict(group=512, tanh=True, pad=8)),
    (1300, 4096, "bf16", "bf16", "token", {}),
    (700, 8192, "fp16", "fp16", "one", {}),
    (620, 8192, "fp32", "fp32", "one", {}),
    # rows at odd addresses through the ring
    (9700, 65, "bf16", "bf16", "token", dict(tanh=True)),
    (4800, 301, "fp16", "fp32", "group", dict(group=700, shift=3)),
    (2400, 1537, "bf16", "bf16", "one", {}),
    (2400, 1030, "fp32", "fp32", "group", dict(group=5, pad=7)),
    (1300, 4001, "bf16", "fp32", "none", dict(pad=2, after=False)),
    (1300, 4095, "fp32", "fp32", "one", dict(before=False)),
    (620, 8191, "fp16", "fp16", "group", dict(group=100)),
    (5000, 77, "bf16", "bf16", "none", dict(block=False)),
]


def norm_case(rows, cols, dtype, wtype, gate, *, group=None, tanh=False, offset=False, pad=0, shift=0, after=True, before=True, block=True,
              weights=True, seed=0):
    import torch
    g = gen(rows, cols, dtype, seed)
    group = {"none": rows, "one": rows, "token": 1, "group": group}[gate]
    after = after and block
    w = lambda: (torch.randn(cols, generator=g) * 0.2 + (0 if offset else 1)).to("cuda", T(wtype))  # noqa: E731
    s = dict(x=rows_tensor(g, rows, cols, dtype, pad, shift, 2.0), y=rows_tensor(g, rows, cols, dtype, pad, shift, 0.5) if block else None,
             w_after=w() if after and weights else None, w_before=w() if before and weights else None,
             gate=rows_tensor(g, -(-rows // group), cols, dtype, pad, shift, 0.7) if gate != "none" and block else None,
             dx_out=rows_tensor(g, rows, cols, dtype, pad, shift, 0.1), dh=rows_tensor(g, rows, cols, dtype, pad, shift, 0.3) if before else None)
    opt = dict(after=after, before=before, offset=offset, tanh=tanh and s["gate"] is not None, alpha=0.7, group_rows=group)
    desc = rb.block_norm(rows, cols, T(dtype), T(wtype), eps=1e-5, alpha=0.7, group_rows=group, norm_after=after, norm_before=before,
                         unit_offset=offset, tanh_gate=opt["tanh"], ld=cols + pad, ld_gate=cols + pad)
    return s, opt, desc


@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_block_norm_forward_and_backward(ctx, case):
    import torch
    rows, cols, dtype, wtype, gate, kw = case
    s, opt, desc = norm_case(rows, cols, dtype, wtype, gate, **kw)
    x_out = like(s["x"]) if s["y"] is not None else None
    h = like(s["x"]) if opt["before"] else None
    rstd = torch.full((rows, 2), 9.0, device="cuda")
    ctx.block_norm_forward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out and x_out[0], h and h[0], rstd)
    ctx.sync()
    want_x, want_h, want_r, size_x, size_h = ref.norm_forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], eps=1e-5, **opt)
    if x_out:
        close(x_out[0], want_x, size_x, dtype, 64, "x_out")
        guarded(x_out)
    if h:
        close(h[0], want_h, size_h, dtype, 64, "h")
        guarded(h)
    close(rstd, want_r, want_r, "fp32", 64, "rstd")
    # backward, from what forward wrote
    x = x_out[0] if x_out else s["x"]
    dx, dy = like(s["x"]), like(s["x"]) if s["y"] is not None else None
    dwa = torch.full((cols,), 9.0, device="cuda") if opt["after"] else None
    dwb = torch.full((cols,), 9.0, device="cuda") if opt["before"] else None
    dg = like(s["gate"]) if s["gate"] is not None else None
    for _ in range(2):                                    # the second call finds the first one's scratch
        ctx.block_norm_backward(desc, x, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], dx[0], dy and dy[0],
                                dwa, dg and dg[0], dwb)
    ctx.sync()
    want = ref.norm_backward(x, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], **opt)
    for name, got, t in (("dx", dx[0], dtype), ("dy", dy and dy[0], dtype), ("dw_after", dwa, "fp32"), ("dgate", dg and dg[0], dtype), ("dw_before", dwb, "fp32")):
        if got is not None:
            close(got, want[name][0], want[name][1], t, 64, name)
    for out in (dx, dy, dg):
        if out is not None:
            guarded(out)


@pytest.mark.parametrize("rows,cols", [(40, 768), (40, 1537), (5000, 768), (5000, 777)])
def test_block_norm_in_place_equals_out_of_place(ctx, rows, cols):
    import torch
    s, opt, desc = norm_case(rows, cols, "bf16", "bf16", "group", group=9)
    x_out, h, rstd = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(rows, 2, device="cuda")
    args = (s["w_after"], s["gate"], s["w_before"])
    ctx.block_norm_forward(desc, s["x"], s["y"], *args, x_out, h, rstd)
    x, y = s["x"].clone(), s["y"].clone()
    ctx.block_norm_forward(desc, x, y, *args, x, y, None)
    ctx.sync()
    assert torch.equal(x, x_out) and torch.equal(y, h)
    grads = [torch.empty_like(s["x"]) for _ in range(2)] + [torch.empty(cols, device="cuda"), torch.empty_like(s["gate"]), torch.empty(cols, device="cuda")]
    ctx.block_norm_backward(desc, x_out, s["y"], *args, rstd, s["dx_out"], s["dh"], *grads)
    dx, dy = s["dx_out"].clone(), s["dh"].clone()
    more = [torch.empty(cols, device="cuda"), torch.empty_like(s["gate"]), torch.empty(cols, device="cuda")]
    ctx.block_norm_backward(desc, x_out, s["y"], *args, rstd, dx, dy, dx, dy, *more)
    ctx.sync()
    for a, b in zip([dx, dy] + more, grads):
        assert torch.equal(a, b)


def test_block_norm_rows_of_zeros_rows_of_nan_and_no_rows(ctx):
    import torch
    s, opt, desc = norm_case(16, 256, "bf16", "bf16", "token")
    s["x"][3], s["y"][3] = 0, 0                            # a row of zeros stays one
    s["x"][5, 7] = float("nan")                            # a NaN stays in its row
    s["y"][6, 9] = float("inf")
    x_out, h, rstd = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(16, 2, device="cuda")
    ctx.block_norm_forward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out, h, rstd)
    ctx.sync()
    assert (x_out[3] == 0).all() and (h[3] == 0).all() and torch.isfinite(rstd[3]).all()
    rest = [r for r in range(16) if r not in (5, 6)]
    assert torch.isfinite(h[rest].float()).all() and torch.isnan(h[5].float()).all() and torch.isnan(x_out[5].float()).sum() == 1
    empty = rb.block_norm(0, 256, torch.bfloat16)
    dwa, dwb = torch.ones(256, device="cuda"), torch.ones(256, device="cuda")
    ctx.block_norm_forward(empty, s["x"], s["y"], s["w_after"], None, s["w_before"], x_out, h, None)
    ctx.block_norm_backward(empty, x_out, s["y"], s["w_after"], None, s["w_before"], rstd, None, h, x_out, h, dwa, None, dwb)
    ctx.sync()
    assert (dwa == 0).all() and (dwb == 0).all()


def test_block_norm_gradient_without_an_incoming_stream_gradient_and_without_optional_outputs(ctx):
    import torch
    s, opt, desc = norm_case(50, 320, "fp32", "fp32", "group", group=20)
    x_out, h, rstd = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(50, 2, device="cuda")
    ctx.block_norm_forward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out, h, rstd)
    dx, dy = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    ctx.block_norm_backward(desc, x_out, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, None, s["dh"], dx, dy)
    ctx.sync()
    want = ref.norm_backward(x_out, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, None, s["dh"], **opt)
    close(dx, *want["dx"], "fp32", 64, "dx")
    close(dy, *want["dy"], "fp32", 64, "dy")


def test_block_norm_gradients_are_the_slopes_of_the_forward_pass(ctx):
    """Central differences of sum(a x_out + b h) along random directions, in single precision: step 2^-7, so the
    third-derivative term is below 2^-14 relative and the rounding 2^-24 2^7 = 2^-17 of the terms' size."""
    import torch
    s, opt, desc = norm_case(12, 200, "fp32", "fp32", "group", group=5, tanh=True)
    a, b = s["dx_out"].double(), s["dh"].double()

    def value(**kw):
        t = {**s, **kw}
        x_out, h = torch.empty(12, 200, device="cuda"), torch.empty(12, 200, device="cuda")
        ctx.block_norm_forward(desc, t["x"], t["y"], t["w_after"], t["gate"], t["w_before"], x_out, h)
        ctx.sync()
        return float((a * x_out.double() + b * h.double()).sum())

    x_out, h, rstd = torch.empty(12, 200, device="cuda"), torch.empty(12, 200, device="cuda"), torch.empty(12, 2, device="cuda")
    ctx.block_norm_forward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], x_out, h, rstd)
    got = dict(x=torch.empty_like(x_out), y=torch.empty_like(x_out), w_after=torch.empty(200, device="cuda"), gate=torch.empty_like(s["gate"]),
               w_before=torch.empty(200, device="cuda"))
    ctx.block_norm_backward(desc, x_out, s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], got["x"], got["y"],
                            got["w_after"], got["gate"], got["w_before"])
    ctx.sync()
    for name, grad in got.items():
        d = torch.sign(grad)                              # every term of the directional slope counts the same way
        step = 2.0 ** -7 if name != "y" else 2.0 ** -9    # y is the smaller tensor
        slope = (value(**{name: s[name] + step * d}) - value(**{name: s[name] - step * d})) / (2 * step)
        want = float(grad.double().abs().sum())
        assert abs(slope - want) <= 2.0 ** -9 * want, (name, slope, want)


# ---------------------------------------------------------------------------------------------------------- router

ROUTER_CASES = [
    # rows, experts, k, dtype, options
    (1, 1, 1, "fp32", {}),
    (1, 8, 2, "bf16", {}),
    (100, 2, 2, "bf16", dict(renorm=True)),
    (333, 7, 3, "fp32", dict(pad=1, masked=20)),
    (512, 8, 2, "bf16", {}),
    (700, 60, 4, "fp32", dict(pad=1, masked=11, closed=5)),
    (257, 64, 6, "fp16", dict(group=100, renorm=True)),
    (90, 100, 8, "bf16", dict(group=1)),
    (400, 128, 8, "fp32", dict(group=64, masked=30, renorm=True)),
    (150, 130, 1, "fp32", dict(shift=1)),
    (300, 256, 8, "bf16", dict(renorm=True)),
    (40, 300, 8, "fp16", dict(group=7, closed=296)),
    (64, 512, 32, "bf16", dict(renorm=True, closed=490)),
    (20, 777, 5, "fp32", {}),
    (16, 1024, 32, "bf16", dict(group=5)),
    (5000, 16, 2, "bf16", dict(group=1250, masked=2000)),
    (64, 32, 4, "bf16", dict(masked=64)),
    # groups so many that a warp takes each, and that they are counted beforehand in the backward pass
    (9600, 24, 3, "fp32", dict(group=2, masked=50)),
    (12000, 256, 2, "bf16", dict(group=3, renorm=True)),
]


def router_case(rows, experts, k, dtype, *, group=None, masked=0, closed=0, renorm=False, pad=0, shift=0, seed=0):
    import torch
    g = gen(rows, experts, k, seed)
    z = rows_tensor(g, rows, experts, dtype, pad, shift, 1.5)
    z.copy_((z.float() * 4).round() / 4)                  # many equal logits
    if closed:
        z[:, torch.randperm(experts, generator=g)[:closed].cuda()] = NINF
    mask = None
    if masked:
        mask = torch.ones(rows, dtype=torch.uint8, device="cuda")
        at = torch.randperm(rows, generator=g)[:masked].cuda()
        mask[at] = 0
        z[at] = float("nan")
    if rows > 10:
        z[rows // 2] = NINF                               # a row that nothing is open for
    group = group or rows
    opt = dict(group_rows=group, coef=0.3, renorm=renorm)
    return z, mask, opt, rb.router(rows, experts, k, T(dtype), ld=experts + pad, **opt)


def router_outputs(rows, experts, k, groups):
    import torch
    i = dict(dtype=torch.int32, device="cuda")
    return dict(index=torch.full((rows, k), 9, **i), weight=torch.full((rows, k), 9.0, device="cuda"), counts=torch.full((groups, experts), 9, **i),
                prob_sum=torch.full((groups, experts), 9.0, device="cuda"), valid=torch.full((groups,), 9, **i), loss=torch.full((1,), 9.0, device="cuda"))


@pytest.mark.parametrize("case", ROUTER_CASES, ids=lambda c: "-".join(map(str, c[:4])))
def test_router_forward_and_backward(ctx, case):
    import torch
    rows, experts, k, dtype, kw = case
    z, mask, opt, desc = router_case(rows, experts, k, dtype, **kw)
    o = router_outputs(rows, experts, k, -(-rows // opt["group_rows"]))
    for _ in range(2):                                    # the arrival counters are as they were after a call
        ctx.router_forward(desc, z, mask, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    ctx.sync()
    want = ref.router_forward(z, mask, k, **opt)
    for name in ("index", "counts", "valid"):
        assert torch.equal(o[name].cpu().long(), want[name]), name
    close(o["weight"], want["weight"], want["weight"], "fp32", 32, "weight")
    close(o["prob_sum"], want["prob_sum"], want["prob_sum"], "fp32", 64, "prob_sum")
    loss = torch.tensor([want["loss"]], dtype=torch.float64)
    close(o["loss"], loss, loss.abs(), "fp32", 64, "loss")
    dweight = torch.randn(rows, k, generator=gen(1, rows)).cuda()
    dloss = torch.tensor([1.5], device="cuda")
    for dl, dw in ((dloss, dweight), (None, None)):
        out = like(z)
        ctx.router_backward(desc, z, o["index"], o["weight"], o["counts"], o["valid"], dl, dw, out[0])
        ctx.sync()
        dz, size = ref.router_backward(want, k, 1.5 if dl is not None else 1.0, dw, **opt)
        close(out[0], dz, size, dtype, 64, "dlogits")
        guarded(out)


def test_router_repeats_itself_and_takes_its_output_over_its_input(ctx):
    import torch
    z, mask, opt, desc = router_case(4000, 128, 8, "bf16", group=500, masked=100)
    a, b = router_outputs(4000, 128, 8, 8), router_outputs(4000, 128, 8, 8)
    for o in (a, b):
        ctx.router_forward(desc, z, mask, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    out = torch.empty_like(z)
    dw = torch.randn(4000, 8, device="cuda")
    ctx.router_backward(desc, z, a["index"], a["weight"], a["counts"], a["valid"], None, dw, out)
    ctx.router_backward(desc, z, a["index"], a["weight"], a["counts"], a["valid"], None, dw, z)
    ctx.sync()
    for name in a:
        assert torch.equal(a[name], b[name]), name
    assert torch.equal(z, out)


@pytest.mark.parametrize("dtype,experts", [("bf16", 16), ("fp32", 128), ("fp32", 300), ("fp16", 7)])
def test_router_never_chooses_nan_and_keeps_near_ties_in_order(ctx, dtype, experts):
    """Logits that differ in their last bit only are chosen in their order, equal ones (0 and -0 among them) by index; a NaN
    is never chosen and spoils its own row's weights, its group's sums and the loss, not the choice."""
    import torch
    z = torch.zeros(6, experts)
    if dtype == "fp32":
        z[0] = torch.nextafter(torch.tensor(1.0), torch.tensor(2.0))
        z[0, 3:] = 1.0
        z[0, 5] = 1.0 + 2.0 ** -21
    z[1, ::2] = -0.0
    z[2, 1] = float("nan")
    z[2, 4] = 2.0
    z[3, 0] = -float("nan")
    z[4] = -torch.arange(experts) - 1.0
    z = z.to(T(dtype)).cuda()
    k = 5
    o = router_outputs(6, experts, k, 2)
    ctx.router_forward(rb.router(6, experts, k, T(dtype), group_rows=3), z, None, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    ctx.sync()
    clean = torch.where(torch.isnan(z), NINF, z.float())
    want = ref.router_forward(clean, None, k, group_rows=3, coef=0.01, renorm=False)
    assert torch.equal(o["index"].cpu().long(), want["index"]) and torch.equal(o["counts"].cpu().long(), want["counts"])
    weight = o["weight"].cpu()
    assert torch.isnan(weight[[2, 3]]).all() and torch.isfinite(weight[[0, 1, 4, 5]]).all() and torch.isnan(o["loss"]).all()


def test_router_gradient_is_the_slope_of_the_loss(ctx):
    """Central differences of loss + sum(d weight) with the choice held: step 2^-8 on logits that are far apart, so that
    no order changes; truncation 2^-16, rounding 2^-24 2^8 = 2^-16 of the value, against a slope of its size / 8."""
    import torch
    rows, experts, k = 32, 16, 3
    g = gen(5)
    z = torch.stack([torch.randperm(experts, generator=g) for _ in range(rows)]).float().cuda() * 0.25
    d = torch.randn(rows, k, generator=g).cuda()
    for renorm in (False, True):
        desc = rb.router(rows, experts, k, torch.float32, group_rows=8, coef=2.0, renorm=renorm)

        def value(t):
            o = router_outputs(rows, experts, k, 4)
            ctx.router_forward(desc, t, None, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
            ctx.sync()
            return float(o["loss"].double() + (o["weight"].double() * d.double()).sum()), o

        _, o = value(z)
        out = torch.empty_like(z)
        ctx.router_backward(desc, z, o["index"], o["weight"], o["counts"], o["valid"], None, d, out)
        ctx.sync()
        step = 2.0 ** -8
        direction = torch.sign(out)
        slope = (value(z + step * direction)[0] - value(z - step * direction)[0]) / (2 * step)
        want = float(out.double().abs().sum())
        assert abs(slope - want) <= 2.0 ** -9 * want


# --------------------------------------------------------------------------------------------------------- distill

DISTILL_CASES = [
    # rows, vocab, k, dtype, ttype, options
    (1, 1, 1, "fp32", "fp32", {}),
    (3, 5, 4, "bf16", "bf16", dict(temperature=2.0)),
    (7, 63, 9, "fp16", "fp32", dict(pad=1)),
    (40, 1000, 64, "bf16", "fp32", dict(temperature=0.7, padded=5)),
    (9, 4097, 20, "fp32", "fp32", dict(shift=1, padded=2)),
    (5, 32000, 1024, "bf16", "fp16", dict(temperature=3.0)),
    (6, 50257, 20, "bf16", "fp32", dict(padded=1)),
    (4, 50257, 20, "fp16", "fp16", dict(pad=7, shift=3)),
    (2, 131072, 64, "fp32", "fp32", {}),
    (2, 140001, 64, "fp32", "fp32", dict(pad=2)),
    (2, 262143, 64, "bf16", "fp32", {}),
    (1, 270001, 100, "bf16", "fp32", dict(temperature=1.5)),
    (600, 200, 16, "bf16", "fp32", dict(padded=300)),
    (350, 4100, 8, "fp32", "fp32", {}),
    # rows enough for the clusters that stay: one, two, five and eight blocks a row
    (1500, 203, 7, "fp32", "fp32", dict(padded=4)),
    (2100, 1003, 20, "bf16", "fp32", dict(padded=100, shift=5)),
    (1400, 16384, 9, "bf16", "bf16", {}),
    (720, 20011, 33, "fp16", "fp32", dict(temperature=2.0)),
    (110, 140001, 64, "bf16", "fp32", dict(padded=3)),
    (170, 128000, 64, "bf16", "fp32", dict(temperature=0.5)),
    (100, 70001, 1024, "fp32", "fp16", dict(pad=3)),
]


def distill_case(rows, vocab, k, dtype, ttype, *, temperature=1.0, padded=0, pad=0, shift=0, seed=0):
    import torch
    g = gen(rows, vocab, k, seed)
    z = rows_tensor(g, rows, vocab, dtype, pad, shift, 2.5)
    index = torch.stack([torch.randperm(vocab, generator=g)[:k] if vocab >= k else torch.randint(0, vocab, (k,), generator=g) for _ in range(rows)]).int().cuda()
    teacher = (torch.randn(rows, k, generator=g) * 2 + 9).to("cuda", T(ttype))
    if k > 3 and rows > 2:
        index[1, 2] = -1                                   # entries that do not take part
        index[1, 3] = vocab
        teacher[2, 1] = NINF
        index[0, 3] = index[0, 0]                          # a doubled entry
    if vocab > 8 and rows > 2:
        z[2, 4:7] = NINF                                   # masked vocabulary
    if padded:
        index[rows - padded:] = -1
        z[rows - padded:] = float("nan")
    return z, index, teacher, rb.distill(rows, vocab, k, T(dtype), T(ttype), temperature=temperature, ld=vocab + pad)


@pytest.mark.parametrize("case", DISTILL_CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_distill_forward_backward_and_step(ctx, case):
    import torch
    rows, vocab, k, dtype, ttype, kw = case
    z, index, teacher, desc = distill_case(rows, vocab, k, dtype, ttype, **kw)
    up = (torch.rand(rows, generator=gen(2, rows)) + 0.5).cuda()
    want = ref.distill(z, index, teacher, kw.get("temperature", 1.0), up)
    f = lambda: torch.full((rows,), 9.0, device="cuda")  # noqa: E731
    loss, lse, loss2, lse2 = f(), f(), f(), f()
    ctx.distill_forward(desc, z, index, teacher, loss, lse)
    back, both = like(z), like(z)
    ctx.distill_backward(desc, z, index, teacher, lse, up, back[0])
    ctx.distill_step(desc, z, index, teacher, up, loss2, lse2, both[0])
    ctx.sync()
    for name, got, t in (("loss", loss, "fp32"), ("lse", lse, "fp32"), ("loss", loss2, "fp32"), ("lse", lse2, "fp32"), ("dz", back[0], dtype), ("dz", both[0], dtype)):
        close(got, want[name], want["s_" + name], t, 96, name)
    guarded(back)
    guarded(both)
    alone = f()
    ctx.distill_forward(desc, z, index, teacher, alone)    # without the log-sum
    ctx.sync()
    assert torch.equal(alone, loss)


@pytest.mark.parametrize("rows,vocab", [(6, 4096), (6, 5001), (6, 140001), (700, 20011)])
def test_distill_writes_the_gradient_over_the_logits(ctx, rows, vocab):
    import torch
    z, index, teacher, desc = distill_case(rows, vocab, 16, "bf16" if vocab < 90000 else "fp32", "fp32", padded=1)
    f = lambda: torch.empty(rows, device="cuda")  # noqa: E731
    loss, lse, out = f(), f(), torch.empty_like(z)
    ctx.distill_step(desc, z, index, teacher, None, loss, lse, out)
    z1, z2 = z.clone(), z.clone()
    ctx.distill_step(desc, z1, index, teacher, None, f(), f(), z1)
    ctx.distill_backward(desc, z, index, teacher, lse, None, out2 := torch.empty_like(z))
    ctx.distill_backward(desc, z2, index, teacher, lse, None, z2)
    ctx.sync()
    assert torch.equal(z1, out) and torch.equal(z2, out2)


def test_distill_rows_without_anything_left(ctx):
    """A student that rules out every logit, or the one the teacher wants: the loss is infinite, the gradient is not."""
    import torch
    z = torch.zeros(3, 100, device="cuda")
    z[0] = NINF
    z[1, 5] = NINF
    index = torch.tensor([[5, 6], [5, 6], [5, 6]], dtype=torch.int32, device="cuda")
    teacher = torch.tensor([[1.0, 0.0]] * 3, device="cuda")
    desc = rb.distill(3, 100, 2, torch.float32)
    loss, lse, dz = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, 100, device="cuda")
    ctx.distill_step(desc, z, index, teacher, None, loss, lse, dz)
    ctx.sync()
    want = ref.distill(z, index, teacher, 1.0)
    assert loss[0] == float("inf") and loss[1] == float("inf") and torch.isfinite(loss[2]) and lse[0] == NINF
    close(dz, want["dz"], want["s_dz"], "fp32", 96, "dz")


def test_distill_gradient_is_the_slope_of_the_loss(ctx):
    """Central differences along the gradient's signs, step 2^-6: truncation 2^-12 / 6 relative, rounding 2^-22 2^6 of the
    loss's terms."""
    import torch
    z, index, teacher, desc = distill_case(8, 300, 12, "fp32", "fp32", temperature=2.0)
    z[2, 4:7] = 0
    f = lambda: torch.empty(8, device="cuda")  # noqa: E731
    dz = torch.empty_like(z)
    ctx.distill_step(desc, z, index, teacher, None, f(), f(), dz)

    def value(t):
        loss = f()
        ctx.distill_forward(desc, t, index, teacher, loss)
        ctx.sync()
        return loss.double().cpu()

    step = 2.0 ** -6
    d = torch.sign(dz)
    slope = (value(z + step * d) - value(z - step * d)) / (2 * step)
    want = dz.double().abs().sum(1).cpu()
    assert ((slope - want).abs() <= 2.0 ** -9 * want).all()


# ------------------------------------------------------------------------------------------- streams and refusals

def test_a_context_works_on_its_own_stream():
    import torch
    stream = torch.cuda.Stream()
    c = rb.Context(workloads.ENV, device=0, stream=stream.cuda_stream)
    z, index, teacher, desc = distill_case(16, 3001, 8, "bf16", "fp32")
    want = ref.distill(z, index, teacher, 1.0)
    loss = torch.zeros(16, device="cuda")
    torch.cuda.synchronize()
    c.distill_forward(desc, z, index, teacher, loss)
    c.sync()
    close(loss, want["loss"], want["s_loss"], "fp32", 96, "loss")
    c.close()


def test_offsets_beyond_32_bits(ctx):
    """Rows whose elements lie more than 2^31 elements behind the first: 40,000 rows 60,000 elements apart."""
    import torch
    rows, cols, ld = 40000, 64, 60000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (rows, cols), (ld, 1))
    x.copy_(torch.randn(rows, cols, device="cuda"))
    h, rstd = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, 2, device="cuda")
    desc = rb.block_norm(rows, cols, torch.bfloat16, norm_after=False, ld_x=ld, ld_y=cols, ld_h=cols)
    ctx.block_norm_forward(desc, x, None, None, None, None, None, h, rstd)
    ctx.sync()
    v = x[-3:].double().cpu()
    want = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)
    close(h[-3:], want, want.abs(), "bf16", 64, "h")
    z = torch.as_strided(buf, (rows, 50), (ld, 1), 1)
    index = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    teacher = torch.zeros(rows, 1, device="cuda")
    loss = torch.empty(rows, device="cuda")
    ctx.distill_forward(rb.distill(rows, 50, 1, torch.bfloat16, torch.float32, ld=ld), z, index, teacher, loss)
    ctx.sync()
    w = ref.distill(z[-3:], index[-3:], teacher[-3:], 1.0)
    close(loss[-3:], w["loss"], w["s_loss"], "fp32", 96, "loss")


def refused(call, *words):
    with pytest.raises(rb.RubickError) as e:
        call()
    assert e.value.code == rb.EINVAL
    for w in words:
        assert w in str(e.value)


def test_refusals(ctx):
    import torch
    b = lambda *s: torch.full(s, 5.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.full(s, 5.0, device="cuda")  # noqa: E731
    i = lambda *s: torch.full(s, 5, dtype=torch.int32, device="cuda")  # noqa: E731
    x, y, w, g, h = b(4, 8), b(4, 8), b(8), b(1, 8), b(4, 8)
    bf = torch.bfloat16

    def norm(desc, *a):
        return lambda: ctx.block_norm_forward(desc, *a)

    ok = (x, y, w, g, w, x, h)
    refused(norm(rb.block_norm(-1, 8, bf), *ok), "rows")
    refused(norm(rb.block_norm(4, 0, bf), *ok), "cols")
    refused(norm(rb.block_norm(4, 16385, bf, ld=16385), *ok), "cols")
    refused(norm(rb.block_norm(4, 8, 7), *ok), "type")
    refused(norm(rb.block_norm(4, 8, bf, torch.float16), *ok), "16-bit")
    refused(norm(rb.block_norm(4, 8, bf, eps=0.0), *ok), "eps")
    refused(norm(rb.block_norm(4, 8, bf, eps=float("nan")), *ok), "eps")
    refused(norm(rb.block_norm(4, 8, bf, alpha=float("inf")), *ok), "alpha")
    refused(norm(rb.block_norm(4, 8, bf, ld=7), *ok), "distance")
    refused(norm(rb.block_norm(4, 8, bf, ld_gate=7), *ok), "ld_gate")
    refused(norm(rb.block_norm(4, 8, bf, group_rows=0), *ok), "group_rows")
    refused(norm(rb.block_norm(4, 8, bf, tanh_gate=True), x, y, w, None, w, x, h), "tanh")
    refused(norm(rb.block_norm(4, 8, bf, norm_after=False), *ok), "not taken")
    refused(norm(rb.block_norm(4, 8, bf), x, y, w, g, w, x, None))
    refused(norm(rb.block_norm(4, 8, bf), x, y, w, g, w, None, h))
    refused(norm(rb.block_norm(4, 8, bf), None, y, w, g, w, x, h))
    refused(norm(rb.block_norm(4, 8, bf), x, None, None, None, w, None, h), "without y")
    bad = rb.block_norm(4, 8, bf)
    bad.flags |= 64
    refused(norm(bad, *ok), "flag")
    d = rb.block_norm(4, 8, bf)
    refused(lambda: ctx.block_norm_backward(d, x, y, w, None, w, f(4, 2), x, h, x, y, f(8), g, f(8)), "not there")
    refused(lambda: ctx.block_norm_backward(d, x, y, w, g, w, None, x, h, x, y), "rstd")
    refused(lambda: ctx.block_norm_backward(d, x, y, w, g, w, f(4, 2), x, None, x, y))
    refused(lambda: ctx.block_norm_backward(d, x, y, w, g, w, f(4, 2), x, h, x, None))

    z, idx, wt, cn, ps, va, lo = b(4, 8), i(4, 2), f(4, 2), i(1, 8), f(1, 8), i(1), f(1)

    def route(desc, *a):
        return lambda: ctx.router_forward(desc, *a)

    ok = (z, None, idx, wt, cn, ps, va, lo)
    refused(route(rb.router(-1, 8, 2, bf), *ok), "rows")
    refused(route(rb.router(4, 0, 2, bf), *ok), "experts")
    refused(route(rb.router(4, 1025, 2, bf), *ok), "experts")
    refused(route(rb.router(4, 8, 0, bf), *ok), "k out")
    refused(route(rb.router(4, 8, 9, bf), *ok), "k out")
    refused(route(rb.router(4, 64, 33, bf), *ok), "k out")
    refused(route(rb.router(4, 8, 2, 9), *ok), "type")
    refused(route(rb.router(4, 8, 2, bf, ld=7), *ok), "ld")
    refused(route(rb.router(4, 8, 2, bf, group_rows=0), *ok), "group_rows")
    refused(route(rb.router(4, 8, 2, bf, coef=float("nan")), *ok), "coef")
    refused(route(rb.router(4, 8, 2, bf), None, None, idx, wt, cn, ps, va, lo), "null")
    refused(route(rb.router(4, 8, 2, bf), z, None, idx, wt, cn, ps, va, None), "loss")
    refused(lambda: ctx.router_backward(rb.router(4, 8, 2, bf), z, idx, wt, cn, None, None, None, z), "null")

    loss, lse, t = f(4), f(4), f(4, 2)

    def dist(desc, *a):
        return lambda: ctx.distill_forward(desc, *a)

    ok = (z, idx, t, loss, lse)
    refused(dist(rb.distill(-1, 8, 2, bf, torch.float32), *ok), "rows")
    refused(dist(rb.distill(4, 0, 2, bf, torch.float32), *ok), "vocab")
    refused(dist(rb.distill(4, 8, 0, bf, torch.float32), *ok), "k out")
    refused(dist(rb.distill(4, 8, 1025, bf, torch.float32), *ok), "k out")
    refused(dist(rb.distill(4, 8, 2, bf, 5), *ok), "type")
    refused(dist(rb.distill(4, 8, 2, bf, torch.float32, ld=7), *ok), "ld")
    for temperature in (0.0, -1.0, float("nan"), float("inf")):
        refused(dist(rb.distill(4, 8, 2, bf, torch.float32, temperature=temperature), *ok), "temperature")
    d = rb.distill(4, 8, 2, bf, torch.float32)
    refused(dist(d, z, idx, t, None, lse), "null")
    refused(lambda: ctx.distill_backward(d, z, idx, t, None, None, z), "null")
    refused(lambda: ctx.distill_step(d, z, idx, t, None, loss, None, z), "null")
    ctx.sync()
    for v in (x, y, w, g, h, z, idx, wt, cn, ps, lo, loss, lse):   # a refused call writes nothing
        assert (v == 5).all()
    with pytest.raises(ValueError):
        rb.router(4, 8, 2, torch.float64)


def test_no_rows(ctx):
    import torch
    loss = torch.ones(1, device="cuda")
    ctx.router_forward(rb.router(0, 8, 2, torch.float32), None, None, None, None, None, None, None, loss)
    ctx.router_backward(rb.router(0, 8, 2, torch.float32), None, None, None, None, None, None, None, None)
    ctx.distill_forward(rb.distill(0, 8, 2, torch.float32), None, None, None, None, None)
    ctx.distill_backward(rb.distill(0, 8, 2, torch.float32), None, None, None, None, None, None)
    ctx.distill_step(rb.distill(0, 8, 2, torch.float32), None, None, None, None, None, None, None)
    ctx.sync()
    assert float(loss) == 0.0
