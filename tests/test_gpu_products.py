"""Linear layers, dropout and the head's cross entropy against double precision.

Tolerances, fixed beforehand.  A result of type T may be off by its rounding, u |want| with u = 2^-8 (bf16), 2^-11 (fp16,
and 2^-24 where it is subnormal), 2^-23 (fp32), plus C 2^-24 times the size of the terms it was summed from, with
C = 2 K + 256 for K products: each addition to a single-precision sum is off by one unit of its last place at most (2^-23 of
the sum, if it is cut off instead of rounded), and the epilogue adds some dozen roundings and an approximated exponential.
A gradient through dz adds half a step of T for every dz, which is rounded between the two products: u times the size of its
terms; a head's step adds another where dz is made of exponentials that were rounded as well.
Dropout chooses the same elements, so it is off by its roundings alone (C = 4)."""
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
from paper_2408_08586_b200 import workloads
from test_gpu_train_ops import T, U, gen, guarded, like, rows_tensor
import product_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]


@pytest.fixture(scope="module")
def ctx():
    return rb.Context(workloads.ENV, device=0)


def close(got, want, bound, dtype, what):
    import torch
    got, want = got.detach().double().to(want.device).reshape(want.shape), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got[~fine]), torch.isnan(want[~fine])), what
    bound = U[dtype] * want.abs() + bound + (2.0 ** -24 if dtype == "fp16" else 1e-37)
    off = ((got - want).abs() / bound)[fine]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} of the tolerance"


def seed_of(a=0x0123456789abcdef, b=(7 << 32) + 5):
    import torch
    return torch.tensor([a, b], dtype=torch.int64, device="cuda")


SEED = (0x0123456789abcdef, (7 << 32) + 5)


# -------------------------------------------------------------------------------------------------------- dropout

def test_the_generator_is_the_published_one(ctx):
    """Known answers of the paper's test vectors, and the kernel's choice word by word."""
    import torch
    assert ref.philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert ref.philox((ref.MASK,) * 4, (ref.MASK,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    x = torch.ones(5, 30, device="cuda")
    out = torch.empty_like(x)
    ctx.dropout_forward(rb.dropout(5, 30, torch.float32, p=0.25), seed_of(), x, None, out)
    for row in range(5):
        for col in range(30):
            word = ref.philox((col // 4, row, SEED[1] & ref.MASK, SEED[1] >> 32), (SEED[0] & ref.MASK, SEED[0] >> 32))[col % 4]
            assert float(out[row, col]) == (1 / 0.75 if word >= 1 << 30 else 0.0) or abs(float(out[row, col]) - 1 / 0.75) < 2.0 ** -22 and word >= 1 << 30


DROPOUT_CASES = [
    # rows, cols, dtype, p, residual, pad, shift
    (1, 1, "fp32", 0.5, False, 0, 0), (1, 4096, "bf16", 0.1, True, 0, 0), (7, 5, "fp16", 0.3, True, 3, 1), (33, 64, "fp16", 0.1, False, 0, 0),
    (130, 97, "bf16", 0.9, True, 0, 0), (64, 257, "fp32", 0.5, True, 3, 2), (1000, 1537, "bf16", 0.1, True, 0, 0), (300, 8192, "fp32", 0.2, False, 8, 0),
    (20, 66, "bf16", 0.0, True, 0, 0), (3000, 130, "fp16", 0.999, False, 2, 0),
]


@pytest.mark.parametrize("rows,cols,dtype,p,residual,pad,shift", DROPOUT_CASES)
def test_dropout(ctx, rows, cols, dtype, p, residual, pad, shift):
    import torch
    g = gen("dropout", rows, cols, dtype)
    x, res = rows_tensor(g, rows, cols, dtype, pad, shift), rows_tensor(g, rows, cols, dtype, pad, shift, 3.0) if residual else None
    desc = rb.dropout(rows, cols, T(dtype), p=p, ld=cols + pad)
    keep = ref.keep(SEED, rows, cols, p)
    for back in (False, True):
        out = like(x)
        r = None if back else res
        if back:
            ctx.dropout_backward(desc, seed_of(), x, out[0])
        else:
            ctx.dropout_forward(desc, seed_of(), x, r, out[0])
        want = ref.d64(x) * keep
        size = want.abs()
        if r is not None:
            want, size = want + ref.d64(r), size + ref.d64(r).abs()
        close(out[0], want, 4 * 2.0 ** -24 * size, dtype, "dropout")
        guarded(out)
    if p > 0.05 and rows * cols > 5000:
        share = float((keep == 0).double().mean())
        assert abs(share - p) < 5 * (p * (1 - p) / (rows * cols)) ** 0.5


def test_dropped_elements_are_zero_whatever_they_hold(ctx):
    import torch
    x = torch.full((40, 64), float("nan"), device="cuda")
    x[:, ::2] = float("inf")
    out = torch.empty_like(x)
    ctx.dropout_forward(rb.dropout(40, 64, torch.float32, p=0.5), seed_of(), x, None, out)
    dropped = ref.keep(SEED, 40, 64, 0.5) == 0
    assert (out.cpu()[dropped] == 0).all() and not torch.isfinite(out.cpu()[~dropped]).any()


def test_dropout_in_place_and_with_distances_of_their_own(ctx):
    import torch
    g = gen("in place")
    x, res = rows_tensor(g, 50, 72, "bf16"), rows_tensor(g, 50, 72, "bf16", 8)
    out = rows_tensor(g, 50, 72, "bf16", 5)
    desc = rb.dropout(50, 72, torch.bfloat16, p=0.4, ld_x=72, ld_res=80, ld_out=77)
    ctx.dropout_forward(desc, seed_of(), x, res, out)
    over = res.clone(memory_format=torch.preserve_format)
    same = torch.empty(50, 80, dtype=torch.bfloat16, device="cuda")[:, :72]
    same.copy_(res)
    ctx.dropout_forward(rb.dropout(50, 72, torch.bfloat16, p=0.4, ld_x=72, ld_res=80, ld_out=80), seed_of(), x, same, same)
    assert torch.equal(same, out) and torch.equal(over, res)
    back = torch.empty(50, 72, dtype=torch.bfloat16, device="cuda")
    ctx.dropout_backward(desc, seed_of(), out, back)            # dout lies as out, dx as x
    close(back, ref.d64(out) * ref.keep(SEED, 50, 72, 0.4), 0.0, "bf16", "dx")
    ctx.dropout_backward(rb.dropout(50, 72, torch.bfloat16, p=0.4), seed_of(), back, back)


# ---------------------------------------------------------------------------------------------------------- linear

LINEAR_CASES = [
    # rows, inputs, outputs, dtype, activation, options
    (1, 1, 1, "bf16", "none", {}),
    (1, 64, 256, "bf16", "silu", dict(bias="same")),
    (3, 40, 24, "fp16", "gelu", dict(bias="fp32", by_output=True, residual=True)),
    (4, 512, 1000, "bf16", "none", dict(residual=True, bias="same")),
    (7, 515, 130, "fp16", "relu", dict(bias="same", pad=3, by_output=True)),
    (16, 1024, 384, "fp16", "none", dict(p=0.1, bias="fp32")),
    (17, 96, 128, "bf16", "gelu_tanh", dict(p=0.3, residual=True, bias="same", pre=True)),
    (64, 333, 129, "bf16", "gelu", dict(p=0.5, shift=1, pre=True)),
    (100, 128, 513, "fp16", "silu", dict(pad=8, residual=True)),
    (127, 64, 64, "bf16", "none", dict(by_output=True)),
    (128, 2048, 128, "bf16", "relu", dict(bias="fp32")),
    (129, 65, 257, "fp16", "gelu_tanh", dict(by_output=True, bias="same", pre=True)),
    (200, 615, 1537, "bf16", "silu", dict(by_output=True, pad=1, bias="same")),
    (300, 768, 768, "bf16", "gelu", dict(residual=True, p=0.1, bias="same", pre=True)),
    (513, 256, 640, "fp16", "none", dict(residual=True)),
    (1000, 72, 1288, "bf16", "gelu_tanh", dict(by_output=True)),
    (2100, 520, 264, "bf16", "none", dict(bias="same", residual=True, p=0.2, pad=8)),
]


def linear_case(rows, inputs, outputs, dtype, activation, opt):
    import torch
    g = gen("linear", rows, inputs, outputs, dtype)
    pad, shift, by_output = opt.get("pad", 0), opt.get("shift", 0), opt.get("by_output", False)
    x = rows_tensor(g, rows, inputs, dtype, pad, shift)
    w = rows_tensor(g, *((outputs, inputs) if by_output else (inputs, outputs)), dtype, pad, shift, inputs ** -0.5)
    btype = "fp32" if opt.get("bias") == "fp32" else dtype
    bias = torch.randn(outputs, generator=g).to(T(btype)).cuda() if opt.get("bias") else None
    res = rows_tensor(g, rows, outputs, dtype, pad, shift, 2.0) if opt.get("residual") else None
    dout = rows_tensor(g, rows, outputs, dtype, pad, shift)
    pre = rows_tensor(g, rows, outputs, dtype, pad, shift)
    desc = rb.linear(rows, inputs, outputs, T(dtype), T(btype), activation=activation, p=opt.get("p", 0.0), by_output=by_output,
                     ld_x=inputs + pad, ld_w=w.shape[1] + pad, ld_out=outputs + pad)
    kw = dict(activation=activation, by_output=by_output, seed=SEED, p=opt.get("p", 0.0))
    return desc, kw, x, w, bias, res, pre, dout


@pytest.mark.parametrize("rows,inputs,outputs,dtype,activation,opt", LINEAR_CASES)
def test_linear_forward(ctx, rows, inputs, outputs, dtype, activation, opt):
    desc, kw, x, w, bias, res, pre, _ = linear_case(rows, inputs, outputs, dtype, activation, opt)
    out, kept = like(pre), like(pre) if opt.get("pre") else None
    ctx.linear_forward(desc, x, w, bias, res, seed_of(), kept[0] if kept else None, out[0])
    ctx.sync()
    want, z, size, size_z = ref.linear_forward(x, w, bias, res, **kw)
    C = (2 * inputs + 256) * 2.0 ** -24
    close(out[0], want, C * size, dtype, "out")
    guarded(out)
    if kept:
        close(kept[0], z, C * size_z, dtype, "pre")
        guarded(kept)


@pytest.mark.parametrize("rows,inputs,outputs,dtype,activation,opt", LINEAR_CASES)
def test_linear_backward(ctx, rows, inputs, outputs, dtype, activation, opt):
    import torch
    desc, kw, x, w, _, _, pre, dout = linear_case(rows, inputs, outputs, dtype, activation, opt)
    dx, dw = like(x), like(w)
    dbias = torch.full((outputs,), 5.0, device="cuda")
    z = None if activation == "none" else pre
    ctx.linear_backward(desc, x, w, z, seed_of(), dout, dx[0], dw[0], dbias)
    ctx.sync()
    want = ref.linear_backward(x, w, z, dout, **kw)
    step = U[dtype] + 64 * 2.0 ** -24
    tiny = 2.0 ** -24 if dtype == "fp16" else 0.0               # half a step of a subnormal dz, a term
    close(dbias, want["dbias"][0], (2 * rows + 256) * 2.0 ** -24 * want["dbias"][1], "fp32", "dbias")
    aw = ref.d64(w).abs().sum(0 if opt.get("by_output") else 1)
    ax = ref.d64(x).abs().sum(0)
    close(dx[0], want["dx"][0], (step + (2 * outputs + 256) * 2.0 ** -24) * want["dx"][1] + tiny * aw, dtype, "dx")
    close(dw[0], want["dw"][0], (step + (2 * rows + 256) * 2.0 ** -24) * want["dw"][1] + tiny * (ax if opt.get("by_output") else ax[:, None]), dtype, "dw")
    guarded(dx)
    guarded(dw)
    # each of them alone is the same
    for only in range(3):
        ask = [torch.zeros_like(t) if i == only else None for i, t in enumerate((dx[0], dw[0], dbias))]
        ld = rb.LinearDesc.from_buffer_copy(desc)
        if only < 2:
            ask[only] = like((x, w)[only])[0]
        ctx.linear_backward(ld, x if only == 1 else None, w if only == 0 else None, z, seed_of(), dout, *ask)
        assert torch.equal(ask[only], (dx[0], dw[0], dbias)[only])


def test_linear_gradients_against_differences(ctx):
    """A loss through forward, its gradient through backward: the difference of two forward passes along a direction."""
    import torch
    g = gen("differences")
    rows, inputs, outputs = 40, 64, 48
    draw = lambda *s: torch.randn(*s, generator=g).half().cuda()  # noqa: E731
    x, w, bias, dout = draw(rows, inputs), draw(inputs, outputs) * 0.125, draw(outputs), draw(rows, outputs)
    desc = rb.linear(rows, inputs, outputs, torch.float16, activation="gelu", p=0.2)
    pre, out, dx, dw = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(x), torch.empty_like(w)
    db = torch.empty(outputs, device="cuda")
    ctx.linear_forward(desc, x, w, bias, None, seed_of(), pre, out)
    ctx.linear_backward(desc, x, w, pre, seed_of(), dout, dx, dw, db)
    vx, vw, vb = draw(rows, inputs), draw(inputs, outputs) * 0.125, draw(outputs)
    eps = 2.0 ** -6
    values = []
    for sign in (1, -1):
        o = ref.linear_forward((x.double() + sign * eps * vx.double()), (w.double() + sign * eps * vw.double()), bias.double() + sign * eps * vb.double(),
                               activation="gelu", seed=SEED, p=0.2)[0]
        values.append(float((o * ref.d64(dout)).sum()))
    slope = (values[0] - values[1]) / (2 * eps)
    got = float((dx.double() * vx.double()).sum() + (dw.double() * vw.double()).sum() + (db.double() * vb.double()).sum())
    size = float((dx.double() * vx.double()).abs().sum() + (dw.double() * vw.double()).abs().sum())
    # roundings of dx, dw and pre (2^-11 each and of every dz), and the differences' own error: third derivatives times eps^2
    assert abs(got - slope) <= 2.0 ** -8 * size


LARGE_CASES = [
    # so many tiles, or so long sums, that each way of cutting a product is taken: pairs of blocks with whole and with narrower
    # tiles, the k dealt out to pairs and joined, or to the blocks of a cluster
    (2048, 2560, 1280, "fp16", "none", dict(p=0.1, bias="fp32", residual=True)),
    (4000, 768, 3001, "bf16", "gelu", dict(pad=1, bias="same", residual=True, pre=True)),
    (5000, 1024, 2048, "bf16", "silu", dict(pre=True, by_output=True, p=0.2, bias="fp32")),
    (9000, 520, 776, "fp16", "gelu_tanh", dict(p=0.3, by_output=True)),
    (512, 8192, 256, "bf16", "relu", dict(bias="same", residual=True)),
    (150, 4100, 640, "fp16", "none", dict(by_output=True, residual=True, p=0.5)),
    (1, 7000, 300, "bf16", "gelu", dict(bias="same", residual=True, pre=True)),
    (48, 2000, 5000, "fp16", "silu", dict(by_output=True, p=0.1, pre=True, pad=3)),
    (20000, 96, 64, "bf16", "none", dict(bias="same")),
]


@pytest.fixture
def on_gpu():
    ref.DEVICE = "cuda"
    yield
    ref.DEVICE = "cpu"


@pytest.mark.parametrize("rows,inputs,outputs,dtype,activation,opt", LARGE_CASES)
def test_linear_large(ctx, on_gpu, rows, inputs, outputs, dtype, activation, opt):
    test_linear_forward(ctx, rows, inputs, outputs, dtype, activation, opt)
    test_linear_backward(ctx, rows, inputs, outputs, dtype, activation, opt)


@pytest.mark.parametrize("rows,hidden,vocab,dtype,opt", [
    (600, 768, 30011, "bf16", dict(by_output=True)),            # dz of the exponentials
    (2000, 320, 20000, "fp16", dict(scale=3.0)),                # the logits twice
    (1000, 1030, 9001, "fp16", dict(by_output=True, pad=1, scale=4.0)),
    (20, 2048, 16384, "bf16", {}),
    (60, 700, 40000, "fp16", dict(by_output=True)),
])
def test_head_loss_large(ctx, on_gpu, rows, hidden, vocab, dtype, opt):
    test_head_loss(ctx, rows, hidden, vocab, dtype, opt)


def test_rows_beyond_32_bits(ctx):
    """Tensors of more than 2^31 elements: the last rows are read and written where they are."""
    import torch
    rows, cols = 33000, 65544
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-3:] = 1.0
    ctx.dropout_forward(rb.dropout(rows, cols, torch.bfloat16, p=0.5), seed_of(), x, None, x)
    ctx.sync()
    assert torch.equal(x[-3:].double().cpu(), ref.keep(SEED, 3, cols, 0.5, first_row=rows - 3)) and not x[:-3].any()
    del x
    n, wide = 40000, 60000
    buf = torch.zeros(n, wide, dtype=torch.bfloat16, device="cuda")
    view = buf[:, 100 * 8:100 * 8 + 64]
    view.copy_(torch.randn(n, 64, generator=torch.Generator().manual_seed(3)).cuda())
    out = buf[:, 300 * 8:300 * 8 + 128]
    w = torch.randn(64, 128, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    ctx.linear_forward(rb.linear(n, 64, 128, torch.bfloat16, ld_x=wide, ld_out=wide), view, w, None, None, None, None, out)
    ctx.sync()
    want = view[-500:].double() @ w.double()
    assert float((out[-500:].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-3
    out[:-1].zero_()
    view.zero_()
    out[-1].zero_()
    assert not buf.any()


def test_two_contexts_at_once(ctx):
    """Calls of two contexts on two streams, which take turns on the GPU: each gets its own results."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [rb.Context(workloads.ENV, device=0, stream=s.cuda_stream) for s in streams]
    sets = [linear_case(1500, 1024, 2048, "bf16", "gelu", dict(p=0.1, bias="same", residual=True)), linear_case(40, 2048, 4096, "fp16", "none", dict(by_output=True))]
    wants, outs = [], []
    for desc, _, x, w, bias, res, pre, dout in sets:
        outs.append([[torch.empty_like(pre), torch.empty_like(x), torch.empty_like(w)] for _ in range(2)])
    torch.cuda.synchronize()

    def both(c, i, to):
        desc, _, x, w, bias, res, pre, dout = sets[i]
        c.linear_forward(desc, x, w, bias, res, seed, None, to[0])
        c.linear_backward(desc, x, w, pre if desc.activation else None, seed, dout, to[1], to[2])
    seed = seed_of()
    torch.cuda.synchronize()
    for i in range(2):
        both(ctx, i, outs[i][0])
    ctx.sync()
    for _ in range(20):
        for i, (c, s) in enumerate(zip(contexts, streams)):
            with torch.cuda.stream(s):
                both(c, i, outs[i][1])
    for c in contexts:
        c.sync()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(*outs[i]))
    for c in contexts:
        c.close()


def test_linear_over_the_residual_and_with_infinite_weights(ctx):
    import torch
    g = gen("over")
    x, w, res = rows_tensor(g, 70, 64, "bf16"), rows_tensor(g, 64, 136, "bf16"), rows_tensor(g, 70, 136, "bf16")
    desc = rb.linear(70, 64, 136, torch.bfloat16, activation="relu")
    out = torch.empty_like(res)
    ctx.linear_forward(desc, x, w, None, res, None, None, out)
    same = res.clone()
    ctx.linear_forward(desc, x, w, None, same, None, None, same)
    assert torch.equal(same, out)
    w[3, 5], x[9, 7] = float("inf"), float("nan")
    ctx.linear_forward(desc, x, w, None, res, None, None, same)
    keep = torch.ones(70, 136, dtype=torch.bool, device="cuda")
    keep[9, :] = False
    keep[:, 5] = False
    assert torch.equal(same[keep], out[keep]) and torch.isnan(same[9]).all()
    up = x[:, 3] > 0
    up[9] = False
    assert (same[up, 5] == float("inf")).all()


def test_no_rows(ctx):
    import torch
    desc = rb.linear(0, 64, 24, torch.bfloat16, by_output=True, ld_w=72)
    dw, buf = like(torch.empty(24, 72, dtype=torch.bfloat16, device="cuda")[:, :64])
    db = torch.ones(24, device="cuda")
    ctx.linear_forward(desc, None, None, None, None, None, None, None)
    ctx.linear_backward(desc, None, None, None, None, None, None, dw, db)
    assert (dw == 0).all() and (db == 0).all()
    guarded((dw, buf))
    ctx.dropout_forward(rb.dropout(0, 8, torch.float32, p=0.1), seed_of(), None, None, None)
    head = rb.head_loss(0, 64, 24, torch.bfloat16, by_output=True, ld_w=72)
    dw.fill_(3)
    ctx.head_loss_forward(head, None, None, None, None)
    ctx.head_loss_step(head, None, None, None, None, None, None, None, dw)
    assert (dw == 0).all()
    dw.fill_(3)
    ctx.head_loss_backward(head, None, None, None, None, None, None, dw)
    assert (dw == 0).all()
    guarded((dw, buf))


# ------------------------------------------------------------------------------------------------------------ head

HEAD_CASES = [
    # rows, hidden, vocab, dtype, options
    (1, 1, 1, "bf16", {}),
    (1, 64, 1000, "bf16", dict(by_output=True)),
    (3, 40, 24, "fp16", {}),
    (32, 96, 5001, "bf16", dict(by_output=True)),
    (33, 97, 777, "fp16", dict(pad=3)),
    (65, 64, 128, "bf16", dict(shift=1)),
    (100, 200, 129, "fp16", dict(by_output=True, pad=8, weight=False)),
    (127, 128, 2000, "bf16", dict(scale=6.0)),
    (129, 256, 4099, "fp16", dict(by_output=True, scale=3.0)),
    (300, 72, 3001, "bf16", dict(pad=5)),
    (700, 136, 1500, "bf16", dict(by_output=True)),
]


def head_case(rows, hidden, vocab, dtype, opt):
    import torch
    g = gen("head", rows, hidden, vocab, dtype)
    pad, shift, by_output = opt.get("pad", 0), opt.get("shift", 0), opt.get("by_output", False)
    h = rows_tensor(g, rows, hidden, dtype, pad, shift)
    w = rows_tensor(g, *((vocab, hidden) if by_output else (hidden, vocab)), dtype, pad, shift, opt.get("scale", 2.0) * hidden ** -0.5)
    label = torch.randint(0, vocab, (rows,), generator=g).to(torch.int32)
    if rows > 2:
        label[rows // 2], label[rows - 1] = -100, vocab
        h[rows // 2], h[rows - 1] = float("nan"), float("inf")
        label[0] = vocab - 1
    dloss = (torch.rand(rows, generator=g) + 0.5).cuda() / rows if opt.get("weight", True) else None
    desc = rb.head_loss(rows, hidden, vocab, T(dtype), by_output=by_output, ld_h=hidden + pad, ld_w=w.shape[1] + pad)
    return desc, h, w, label.cuda(), dloss, by_output


def check_head(want, got, rows, hidden, vocab, dtype, dloss, h, w, by_output, roundings=1):
    C = (2 * hidden + 256) * 2.0 ** -24
    live = 0 if dloss is None else float(dloss.max())
    for name in ("loss", "lse"):
        if name in got:
            value, size = want[name]
            close(got[name], value, C * (size + 1) + 64 * 2.0 ** -24, "fp32", name)
    # every dz is rounded: half a step, or (fp16) half a step of a subnormal number under the common power of two
    tiny = (live or 1.0) * 2.0 ** -38
    aw = ref.d64(w).abs().sum(0 if by_output else 1)
    ah = ref.d64(h).abs()
    ah = ah[ah.isfinite().all(1)].sum(0)
    for name, K in (("dh", vocab), ("dw", rows)):
        if got.get(name) is not None:
            value, size, logits = want[name]
            few = tiny * (aw if name == "dh" else ah if by_output else ah[:, None])
            close(got[name], value, (roundings * U[dtype] + (2 * K + 256) * 2.0 ** -24) * size + C * logits + few, dtype, name)


@pytest.mark.parametrize("rows,hidden,vocab,dtype,opt", HEAD_CASES)
def test_head_loss(ctx, rows, hidden, vocab, dtype, opt):
    import torch
    desc, h, w, label, dloss, by_output = head_case(rows, hidden, vocab, dtype, opt)
    want = ref.head(h, w, label, dloss, by_output=by_output)
    f32 = lambda: torch.full((rows,), 9.0, device="cuda")  # noqa: E731
    loss, lse, loss2, lse2 = f32(), f32(), f32(), f32()
    dh, dw, dh2, dw2 = like(h), like(w), like(h), like(w)
    ctx.head_loss_forward(desc, h, w, label, loss, lse)
    ctx.head_loss_backward(desc, h, w, label, lse, dloss, dh[0], dw[0])
    ctx.head_loss_step(desc, h, w, label, dloss, loss2, lse2, dh2[0], dw2[0])
    ctx.sync()
    check_head(want, dict(loss=loss, lse=lse, dh=dh[0], dw=dw[0]), rows, hidden, vocab, dtype, dloss, h, w, by_output)
    check_head(want, dict(loss=loss2, lse=lse2, dh=dh2[0], dw=dw2[0]), rows, hidden, vocab, dtype, dloss, h, w, by_output, roundings=2)
    for out in (dh, dw, dh2, dw2):
        guarded(out)
    if rows > 2:
        for r in (rows // 2, rows - 1):
            assert loss[r] == 0 and lse[r] == 0 and (dh[0][r] == 0).all() and (dh2[0][r] == 0).all()
    # each gradient alone, and without the log-sums
    one, other, l3 = like(h), like(w), f32()
    ctx.head_loss_step(desc, h, w, label, dloss, l3, None, one[0], None)
    ctx.head_loss_backward(desc, h, w, label, lse, dloss, None, other[0])
    assert torch.equal(one[0], dh2[0]) and torch.equal(other[0], dw[0]) and torch.equal(l3, loss2)
    ctx.head_loss_step(desc, h, w, label, dloss, l3, lse2, None, None)
    assert torch.equal(l3, loss2) and torch.equal(lse2, lse)


def test_head_loss_in_pieces_of_the_vocabulary(ctx):
    """So many rows that dz of the whole vocabulary would take more than the 256 MB a piece may have."""
    import torch
    rows, hidden, vocab = 66000, 16, 4500
    desc, h, w, label, dloss, _ = head_case(rows, hidden, vocab, "bf16", dict(scale=1.0))
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    loss = torch.empty(rows, device="cuda")
    ctx.head_loss_step(desc, h, w, label, dloss, loss, None, dh, dw)
    ctx.sync()
    want = ref.head(h, w, label, dloss)
    check_head(want, dict(loss=loss, dh=dh, dw=dw), rows, hidden, vocab, "bf16", dloss, h, w, False)


def test_head_loss_far_from_zero(ctx):
    """Logits that are all large: what counts is their differences.  h = [64, small], w = [64, ..] puts every logit near
    4,096; a common offset changes neither loss nor gradients but by what a single-precision logit can hold."""
    import torch
    g = gen("far")
    rows, hidden, vocab = 50, 64, 600
    h, w = rows_tensor(g, rows, hidden, "bf16"), rows_tensor(g, hidden, vocab, "bf16", scale=0.25)
    h[:, 0], w[0, :] = 64.0, 64.0
    label = torch.randint(0, vocab, (rows,), generator=g).to(torch.int32).cuda()
    desc = rb.head_loss(rows, hidden, vocab, torch.bfloat16)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_loss_step(desc, h, w, label, None, loss, lse, dh, dw)
    check_head(ref.head(h, w, label), dict(loss=loss, lse=lse, dh=dh, dw=dw), rows, hidden, vocab, "bf16", None, h, w, False)


def test_head_loss_with_closed_tokens_and_small_weights(ctx):
    """Logits of -inf (a token whose weights say so), a label on one of them, and loss weights that half precision cannot hold."""
    import torch
    g = gen("closed")
    rows, hidden, vocab = 40, 32, 500
    h, w = rows_tensor(g, rows, hidden, "fp16"), rows_tensor(g, vocab, hidden, "fp16")
    h[:, 0] = 1.0
    w[130:400, 0] = float("-inf")
    label = torch.randint(400, 500, (rows,), generator=g).to(torch.int32)
    label[3] = 200
    dloss = torch.full((rows,), 1e-9, device="cuda")
    desc = rb.head_loss(rows, hidden, vocab, torch.float16, by_output=True)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dw = torch.empty_like(w)
    ctx.head_loss_step(desc, h, w, label.cuda(), dloss, loss, lse, None, dw)
    open_ = torch.cat([w[:130], w[400:]])
    z = h.double() @ open_.double().t()
    want = torch.logsumexp(z, 1).cpu()
    assert float((lse.cpu().double() - want).abs().max()) <= 1e-5
    assert loss[3] == float("inf") and torch.isfinite(loss[torch.arange(rows) != 3]).all()
    p = torch.softmax(z, 1)
    for r in range(rows):
        if r != 3:
            p[r, int(label[r]) - 400 + 130] -= 1
    size = p.t().abs() @ h.double().abs()
    off = (torch.cat([dw[:130], dw[400:]]).double() - 1e-9 * (p.t() @ h.double())).abs()
    assert (dw[130:200] == 0).all()
    assert (off <= 1e-9 * 2.0 ** -10 * size + 2.0 ** -24).all()


def test_head_loss_with_the_largest_weights(ctx):
    """Loss weights near single precision's largest: half precision's gradients overflow to infinities of the right sign, never
    to NaN, and bfloat16's are as exact as others."""
    import torch
    for rows in (20, 40):
        for dtype, weight in (("fp16", 1e38), ("bf16", 1e34)):
            desc, h, w, label, _, _ = head_case(rows, 32, 500, dtype, {})
            dloss = torch.full((rows,), weight, device="cuda")
            loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            dw = torch.empty_like(w)
            ctx.head_loss_step(desc, h, w, label, dloss, loss, lse, None, dw)
            want, size, _ = ref.head(h, w, label, dloss)["dw"]
            got = dw.double().cpu()
            assert not torch.isnan(got).any()
            sure = want.abs() > 2.0 ** -6 * size
            if dtype == "fp16":
                assert (got[sure] == torch.copysign(torch.tensor(float("inf"), dtype=torch.float64), want[sure])).all()
            else:
                assert ((got - want).abs() <= 2.0 ** -7 * (want.abs() + size)).all()


def test_sums_over_millions_of_rows(ctx):
    """2^21 positive products a sum, which tensor memory must not sum in one go: half precision's rounding (2^-11) and what sums of
    131,072 are cut off by at most (8,192 joins of 2^-23 each: 2^-10)."""
    import torch
    rows = 1 << 21
    g = torch.Generator(device="cuda").manual_seed(11)
    x, dout = (torch.rand(rows, n, generator=g, device="cuda").mul_(0.125).half() for n in (24, 72))
    dw = torch.empty(24, 72, dtype=torch.float16, device="cuda")
    ctx.linear_backward(rb.linear(rows, 24, 72, torch.float16), x, dw, None, None, dout, None, dw)
    ctx.sync()
    want = x.double().t() @ dout.double()
    assert float(((dw.double() - want).abs() / want).max()) <= 2.0 ** -11 + 2.0 ** -10


def test_results_do_not_depend_on_what_ran_before(ctx):
    """Twice the same call gives the same bits, with other calls of the context in between."""
    import torch
    desc, h, w, label, dloss, _ = head_case(300, 72, 3001, "bf16", {})
    outs = []
    for _ in range(2):
        loss, lse = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        ctx.head_loss_step(desc, h, w, label, dloss, loss, lse, dh, dw)
        outs.append((loss, lse, dh, dw))
        test_linear_backward(ctx, 513, 256, 640, "fp16", "none", dict(residual=True))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# -------------------------------------------------------------------------------------------------------- refusals

def test_refusals(ctx):
    import torch
    bf = torch.bfloat16
    x, w, o = (torch.zeros(64, 64, dtype=bf, device="cuda") for _ in range(3))
    f = torch.zeros(64, device="cuda")
    lab = torch.zeros(64, dtype=torch.int32, device="cuda")
    launched = rb.kernel_launches()

    def refused(call, *args, code=rb.EINVAL):
        with pytest.raises(rb.RubickError) as e:
            call(*args)
        assert e.value.code == code and len(str(e.value)) > 20

    def changed(desc, **kw):
        for k, v in kw.items():
            setattr(desc, k, v)
        return desc

    lin = lambda **kw: changed(rb.linear(64, 64, 64, bf), **kw)  # noqa: E731
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(inputs=0), dict(outputs=0), dict(outputs=(1 << 24) + 1), dict(dtype=rb.F32), dict(dtype=9), dict(btype=rb.F16),
               dict(flags=2), dict(activation=5), dict(activation=-1), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(reserved=1), dict(ld_x=63), dict(ld_w=63),
               dict(ld_out=63)):
        refused(ctx.linear_forward, lin(**kw), x, w, None, None, seed_of(), None, o)
    refused(ctx.linear_forward, lin(p=0.5), x, w, None, None, None, None, o)                     # no seed
    refused(ctx.linear_forward, lin(ld_res=63), x, w, None, o, None, None, o)
    refused(ctx.linear_forward, lin(ld_pre=63), x, w, None, None, None, o, o)
    for args in ((None, w, None, None, None, None, o), (x, None, None, None, None, None, o), (x, w, None, None, None, None, None)):
        refused(ctx.linear_forward, lin(), *args)
    refused(ctx.linear_backward, lin(activation=1), x, w, None, None, o, x, w, None)             # no pre
    refused(ctx.linear_backward, lin(), x, None, None, None, o, x, None, None)                   # dx without w
    refused(ctx.linear_backward, lin(), None, w, None, None, o, None, w, None)                   # dw without x
    refused(ctx.linear_backward, lin(), x, w, None, None, None, x, w, None)
    refused(ctx.linear_forward, lin(), x.float(), w, None, None, None, None, o)                  # another type
    refused(ctx.linear_forward, lin(), x.t(), w.t(), None, None, None, None, o[:, ::2])
    drop = lambda **kw: changed(rb.dropout(64, 64, bf, p=0.5), **kw)  # noqa: E731
    for kw in (dict(rows=-1), dict(cols=0), dict(dtype=3), dict(p=1.0), dict(p=float("nan")), dict(ld_x=10), dict(ld_out=63), dict(reserved=3)):
        refused(ctx.dropout_forward, drop(**kw), seed_of(), x, None, o)
    refused(ctx.dropout_forward, drop(), None, x, None, o)
    refused(ctx.dropout_forward, drop(ld_res=63), seed_of(), x, x, o)
    refused(ctx.dropout_backward, drop(), seed_of(), x, None)
    refused(ctx.dropout_backward, drop(), seed_of().int(), x, o)
    head = lambda **kw: changed(rb.head_loss(64, 64, 64, bf), **kw)  # noqa: E731
    for kw in (dict(rows=-1), dict(hidden=0), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dtype=rb.F32), dict(flags=4), dict(ld_h=63), dict(ld_w=63)):
        refused(ctx.head_loss_forward, head(**kw), x, w, lab, f)
        refused(ctx.head_loss_step, head(**kw), x, w, lab, f, f, f, o, o)
        refused(ctx.head_loss_backward, head(**kw), x, w, lab, f, f, o, o)
    for args in ((None, w, lab, f), (x, None, lab, f), (x, w, None, f), (x, w, lab, None)):
        refused(ctx.head_loss_forward, head(), *args)
    refused(ctx.head_loss_backward, head(), x, w, lab, None, f, o, o)
    refused(ctx.head_loss_forward, head(), x, w, lab.long(), f)
    with pytest.raises((KeyError, ValueError)):
        rb.linear(4, 4, 4, bf, activation="tanh")
    assert rb.kernel_launches() == launched
