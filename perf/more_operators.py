"""The matrix products, the dropout and the head's loss of a training step, in plain form and through the framework's
entry points.  (The block norm, the router and the distillation loss are in perf/operators.py.)

Three operators (rows are tokens, every size is in elements):

    linear    z = x W + b;  out = residual + drop(act(z)), act one of none, relu, gelu, gelu_tanh, silu;
              backward: dz = act'(z) drop(dout), dx = dz W^T, dW = x^T dz, db = sum of dz over the rows
    dropout   out = residual + drop(x);  backward: dx = drop(dout)
    head      loss = log sum_v exp(z_v) - z_label with z = h W over the vocabulary, 0 for rows without a label;
              backward: dz = g (softmax(z) - onehot(label)), dh = dz W^T, dW = h^T dz

drop(v) = v / (1 - p) where the element is kept, else 0.  Element (row, col) is kept when word col % 4 of Philox4x32-10
(Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) at the counter (col / 4, row, offset, offset's upper
half) under the key seed is at least p 2^32; {seed, offset} lie on the device.  The mask is never stored.

`own = False`: elementary torch operations in 32 bits.  `own = True`: the library's kernels.
"""
import math
import struct

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LOSS_SCALE = 1024.0   # half precision trains under a loss scale: the gradients that come in carry it
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
NINF = float("-inf")


# ---------------------------------------------------------------------------------------------------------- cases

def _dropout(name, back, rows, cols, dtype, **kw):
    c = dict(name=name, op="dropout", back=back, rows=rows, cols=cols, dtype=dtype, p=0.1, residual=False, pad=0)
    c.update(kw)
    return c


def _linear(name, back, rows, inputs, outputs, dtype, **kw):
    c = dict(name=name, op="linear", back=back, rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, btype=dtype, bias=True,
             act="none", p=0.0, residual=False, keep_pre=False, by_output=False, pad=0)
    c.update(kw)
    return c


def _head(name, part, rows, hidden, vocab, dtype, **kw):
    c = dict(name=name, op="head", part=part, rows=rows, hidden=hidden, vocab=vocab, dtype=dtype, by_output=False, padded=0, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # a handful of tokens on their way into the residual stream; latency counts
        _dropout("dropout fwd, 4 tokens", False, 4, 4096, "bf16", residual=True),
        # eight sequences of 2,048 tokens: a block's output joins the residual stream
        _dropout("dropout fwd, 8 sequences", False, 16384, 4096, "bf16", residual=True),
        # the backward pass of a model under test in single precision, odd width, rows cut from a wider buffer
        _dropout("dropout bwd, odd width", True, 3001, 1537, "fp32", p=0.25, pad=3),
        # a handful of tokens through one projection: samples drawn from a model between training steps; latency counts
        _linear("linear fwd, 4 tokens", False, 4, 4096, 4096, "bf16", residual=True),
        # a small batch of an odd width, the weight with a row per output, rows cut from a wider buffer
        _linear("linear fwd, odd width", False, 200, 615, 1537, "bf16", act="silu", by_output=True, pad=1),
        # the way down of a block for one sequence: bias, dropout and the residual stream
        _linear("linear fwd, down", False, 2048, 5120, 1280, "fp16", btype="fp32", p=0.1, residual=True),
        # the way up of a block for four sequences, what the activation's gradient needs is kept
        _linear("linear fwd, up", False, 8192, 4096, 16384, "bf16", act="gelu_tanh", keep_pre=True),
        # the backward pass of a small projection over eight sequences: few weights, many rows
        _linear("linear bwd, 8 sequences", True, 16384, 768, 768, "fp16", act="gelu", p=0.1, by_output=True),
        # the backward pass of a block's way up over two sequences
        _linear("linear bwd, 2 sequences", True, 4096, 2048, 8192, "bf16", act="gelu_tanh", btype="fp32"),
        # an evaluation batch of few rows, the head tied to an embedding of an odd number of tokens
        _head("head fwd, 32 rows", "fwd", 32, 768, 50257, "bf16", by_output=True),
        # the backward pass alone, when the loss is one term of several
        _head("head bwd, 1,000 rows", "bwd", 1000, 2048, 32000, "fp16"),
        # a whole training step of the head: loss and gradients of 2,048 tokens at once, the last ones padding
        _head("head step, 2,048 rows", "step", 2048, 4096, 128000, "bf16", by_output=True, padded=48),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, unit):
    """A size between lo and hi, spread over its logarithm: half the time a multiple of `unit`."""
    n = _log(rng, lo, hi)
    return max(unit, n // unit * unit) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["dropout", "linear", "linear", "head", "head"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 40)])
    p = rng.choice([0.1, 0.1, 0.5, round(rng.uniform(0.0, 0.9), 3)])
    if op == "dropout":
        dtype = rng.choice([dtype, dtype, "fp32"])
        size = 4 if dtype == "fp32" else 2
        cols = _size(rng, 64, 16384, 64)
        rows = _log(rng, 1, min(32768, (1 << 27) // (size * cols)))
        back = rng.random() < 0.4
        c = _dropout("", back, rows, cols, dtype, p=p, residual=not back and rng.random() < 0.6, pad=pad)
    elif op == "linear":
        inputs, outputs = _size(rng, 64, 8192, 64), _size(rng, 64, 16384, 64)
        rows = _log(rng, 1, min(16384, int(1e12 / (2 * inputs * outputs))))
        back = rng.random() < 0.5
        act = rng.choice(ACTS)
        c = _linear("", back, rows, inputs, outputs, dtype, btype=rng.choice([dtype, "fp32"]), bias=rng.random() < 0.7, act=act,
                    p=rng.choice([0.0, p]), residual=not back and rng.random() < 0.5, keep_pre=not back and rng.random() < 0.4,
                    by_output=rng.random() < 0.5, pad=pad)
    else:
        hidden, vocab = _size(rng, 64, 5120, 64), _size(rng, 1000, 150000, 64)
        rows = _log(rng, 1, min(8192, int(1e12 / (2 * hidden * vocab))))
        c = _head("", rng.choice(["fwd", "bwd", "step"]), rows, hidden, vocab, dtype, by_output=rng.random() < 0.5,
                  padded=rng.choice([0, rng.randint(0, rows // 3)]), pad=pad)
    del c["name"]
    return c


def work(case):
    c = case
    b = {"bf16": 2, "fp16": 2, "fp32": 4}
    e, n = b[c["dtype"]], c["rows"]
    if c["op"] == "dropout":
        return {"bytes": n * c["cols"] * e * (2 + c["residual"]) + 16, "flops": n * c["cols"] * (1 + c["residual"])}
    if c["op"] == "linear":
        k, m = c["inputs"], c["outputs"]
        if not c["back"]:
            return {"bytes": e * (n * k + k * m + n * m * (1 + c["residual"] + c["keep_pre"])) + c["bias"] * m * b[c["btype"]], "flops": 2 * n * k * m}
        return {"bytes": e * (2 * n * k + 2 * k * m + n * m * (1 + (c["act"] != "none"))) + c["bias"] * 4 * m, "flops": 4 * n * k * m}
    h, v, live = c["hidden"], c["vocab"], n - c["padded"]
    if c["part"] == "fwd":
        return {"bytes": e * (live * h + h * v) + 12 * n, "flops": 2 * live * h * v}
    # the logits once more (or once), and two products with their gradient
    return {"bytes": 2 * e * (n * h + h * v) + (12 if c["part"] == "bwd" else 16) * n, "flops": 6 * live * h * v}


# --------------------------------------------------------------------------------------------------------- inputs

def _rows(n, cols, pad, dtype):
    """An [n, cols] tensor whose rows are `cols + pad` elements apart."""
    return torch.empty(n, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["dtype"]]
    n, pad = c["rows"], c["pad"]
    s = {"case": c}
    scale = LOSS_SCALE if c["dtype"] == "fp16" else 1.0
    f32 = dict(dtype=torch.float32, device="cuda")

    def normal(rows, cols, scale=1.0, pad=pad):
        v = _rows(rows, cols, pad, t)
        v.copy_(torch.randn(rows, cols, generator=g, device="cuda").mul_(scale))
        return v

    if c["op"] != "head":
        c["p"] = struct.unpack("f", struct.pack("f", c["p"]))[0]          # the probability is a single-precision number
        s["seed"] = torch.randint(-(1 << 62), 1 << 62, (2,), generator=g, device="cuda")
    if c["op"] == "dropout":
        s["x"] = normal(n, c["cols"])
        s["residual"] = normal(n, c["cols"], 3.0) if c["residual"] else None
        s["out"] = {"dx" if c["back"] else "out": _rows(n, c["cols"], pad, t)}
    elif c["op"] == "linear":
        k, m = c["inputs"], c["outputs"]
        s["x"] = normal(n, k)
        s["w"] = normal(m, k, k ** -0.5) if c["by_output"] else normal(k, m, k ** -0.5)
        s["bias"] = torch.randn(m, generator=g, device="cuda").mul_(0.3).to(TYPES[c["btype"]]) if c["bias"] else None
        if c["back"]:
            s["pre"] = normal(n, m) if c["act"] != "none" else None
            s["dout"] = normal(n, m, 0.001 * scale)
            s["out"] = {"dx": _rows(n, k, pad, t), "dw": _rows(*s["w"].shape, pad, t), "dbias": torch.empty(m, **f32) if c["bias"] else None}
        else:
            s["residual"] = normal(n, m, 2.0) if c["residual"] else None
            s["out"] = {"out": _rows(n, m, pad, t), "pre": _rows(n, m, pad, t) if c["keep_pre"] else None}
    else:
        h, v = c["hidden"], c["vocab"]
        s["h"] = x = normal(n, h)
        s["w"] = w = normal(v, h, 2.0 * h ** -0.5) if c["by_output"] else normal(h, v, 2.0 * h ** -0.5)
        label = torch.randint(0, v, (n,), generator=g, device="cuda")
        # a model in training likes some of the labels: their rows lean towards the label's weights
        at = (w[label] if c["by_output"] else w[:, label].t()).float()
        lean = torch.rand(n, 1, generator=g, device="cuda").mul_(3.0)
        x += (lean * at).to(t)
        label[n - c["padded"]:] = -1
        s["label"] = label.to(torch.int32)
        s["weight"] = torch.rand(n, generator=g, device="cuda").add_(0.5) * (scale / n)
        s["lse"] = torch.zeros(n, **f32)
        if c["part"] == "bwd":
            for a in range(0, n, 1024):
                s["lse"][a:a + 1024] = _head_rows(s, a)[1]
            s["lse"][n - c["padded"]:] = 0
        s["out"] = {} if c["part"] == "bwd" else {"loss": torch.empty(n, **f32), "lse": s["lse"]}
        if c["part"] != "fwd":
            s["out"].update(dh=_rows(n, h, pad, t), dw=_rows(*w.shape, pad, t))
    return s


# ---------------------------------------------------------------------------------------------------- plain forms

def _some(d):
    return {k: v for k, v in d.items() if v is not None}


def _words(seed, first, rows, cols):
    """Philox4x32-10 words of the elements of `rows` rows from row `first`, as 64-bit integers."""
    low = 0xFFFFFFFF
    quads = -(-cols // 4)
    key = [seed[0] & low, (seed[0] >> 32) & low]
    col = torch.arange(quads, device="cuda")[None, :].expand(rows, quads)
    row = torch.arange(first, first + rows, device="cuda")[:, None].expand(rows, quads)
    x = [col, row, (seed[1] & low).expand(rows, quads), ((seed[1] >> 32) & low).expand(rows, quads)]
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [((b >> 32) & low) ^ x[1] ^ key[0], b & low, ((a >> 32) & low) ^ x[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    return torch.stack(x, 2).reshape(rows, 4 * quads)[:, :cols]


def _drop(v, s):
    p = s["case"]["p"]
    if p == 0.0:
        return v
    for a in range(0, len(v), 4096):            # (in runs of rows: 64-bit words of a whole tensor would not fit beside it)
        part = v[a:a + 4096]
        part.copy_(torch.where(_words(s["seed"], a, *part.shape) >= int(p * 4294967296.0), part * (1.0 / (1.0 - p)), 0.0))
    return v


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    e = 1.0 / (1.0 + torch.exp(-z))
    return e * (1.0 + z * (1.0 - e))


def _linear_forward(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    w = s["w"].float()
    z = s["x"].float() @ (w.t() if c["by_output"] else w)
    if c["bias"]:
        z += s["bias"].float()
    pre = z.to(t) if c["keep_pre"] else None
    out = _drop(_act(z, c["act"]), s)
    if c["residual"]:
        out = s["residual"].float() + out
    return _some({"out": out.to(t), "pre": pre})


def _linear_backward(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    dz = _drop(s["dout"].float(), s)
    if c["act"] != "none":
        dz = dz * _slope(s["pre"].float(), c["act"])
    x, w = s["x"].float(), s["w"].float()
    return _some({"dx": (dz @ (w if c["by_output"] else w.t())).to(t), "dw": (dz.t() @ x if c["by_output"] else x.t() @ dz).to(t),
                  "dbias": dz.sum(0) if c["bias"] else None})


def _head_rows(s, a, w=None):
    """(logits, lse) of up to 1,024 rows from row a"""
    if w is None:
        w = s["w"].float()
    z = s["h"][a:a + 1024].float() @ (w.t() if s["case"]["by_output"] else w)
    top = z.max(1, keepdim=True)[0]
    return z, (top + (z - top).exp().sum(1, keepdim=True).log())[:, 0]


def _head_plain(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    w = s["w"].float()
    out = {k: torch.empty(c["rows"], dtype=torch.float32, device="cuda") for k in ("loss", "lse")}
    dh, dw = [], torch.zeros_like(w) if c["part"] != "fwd" else None
    for a in range(0, c["rows"], 1024):
        z, lse = _head_rows(s, a, w)
        label = s["label"][a:a + 1024].long()[:, None]
        live = label >= 0
        at = label.clamp(min=0)
        if c["part"] == "bwd":
            lse = s["lse"][a:a + 1024]
        else:
            out["loss"][a:a + 1024] = torch.where(live[:, 0], lse - z.gather(1, at)[:, 0], 0.0)
            out["lse"][a:a + 1024] = torch.where(live[:, 0], lse, 0.0)
        if c["part"] != "fwd":
            dz = (z - lse[:, None]).exp()
            dz.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
            dz = torch.where(live, dz * s["weight"][a:a + 1024, None], 0.0)
            x = torch.where(live, s["h"][a:a + 1024].float(), 0.0)
            dh.append((dz @ (w if c["by_output"] else w.t())).to(t))
            dw += dz.t() @ x if c["by_output"] else x.t() @ dz
    if c["part"] == "bwd":
        out = {}
    if c["part"] != "fwd":
        out.update(dh=torch.cat(dh), dw=dw.to(t))
    return out


# ------------------------------------------------------------------------------------------------------- the run

_context = None


def _ctx():
    """The program's one context, on the stream that torch works on."""
    global _context
    if _context is None:
        from paper_2408_08586_b200 import binding, workloads
        _context = binding.Context(workloads.ENV, stream=torch.cuda.current_stream().cuda_stream)
    return _context


def _plan(s):
    """The descriptor of a state's sizes, made once, as a program with fixed shapes keeps it."""
    if "plan" not in s:
        from paper_2408_08586_b200 import binding
        c = s["case"]
        t, pad = TYPES[c["dtype"]], c["pad"]
        if c["op"] == "dropout":
            s["plan"] = binding.dropout(c["rows"], c["cols"], t, p=c["p"], ld=c["cols"] + pad)
        elif c["op"] == "linear":
            s["plan"] = binding.linear(c["rows"], c["inputs"], c["outputs"], t, TYPES[c["btype"]], activation=c["act"], p=c["p"],
                                       by_output=c["by_output"], ld_x=c["inputs"] + pad, ld_w=s["w"].shape[1] + pad, ld_out=c["outputs"] + pad)
        else:
            s["plan"] = binding.head_loss(c["rows"], c["hidden"], c["vocab"], t, by_output=c["by_output"], ld_h=c["hidden"] + pad,
                                          ld_w=s["w"].shape[1] + pad)
        s["result"] = _some(s["out"])
    return s["plan"]


def run(state):
    s, c = state, state["case"]
    if own:
        ctx, plan, o = _ctx(), _plan(s), s["out"]
        if c["op"] == "dropout":
            if c["back"]:
                ctx.dropout_backward(plan, s["seed"], s["x"], o["dx"])
            else:
                ctx.dropout_forward(plan, s["seed"], s["x"], s["residual"], o["out"])
        elif c["op"] == "linear":
            if c["back"]:
                ctx.linear_backward(plan, s["x"], s["w"], s["pre"], s["seed"], s["dout"], o["dx"], o["dw"], o["dbias"])
            else:
                ctx.linear_forward(plan, s["x"], s["w"], s["bias"], s["residual"], s["seed"], o["pre"], o["out"])
        elif c["part"] == "fwd":
            ctx.head_loss_forward(plan, s["h"], s["w"], s["label"], o["loss"], o["lse"])
        elif c["part"] == "bwd":
            ctx.head_loss_backward(plan, s["h"], s["w"], s["label"], s["lse"], s["weight"], o["dh"], o["dw"])
        else:
            ctx.head_loss_step(plan, s["h"], s["w"], s["label"], s["weight"], o["loss"], o["lse"], o["dh"], o["dw"])
        return s["result"]
    if c["op"] == "dropout":
        v = _drop(s["x"].float().clone(), s)
        if c["residual"]:
            v = s["residual"].float() + v
        return {"dx" if c["back"] else "out": v.to(TYPES[c["dtype"]])}
    if c["op"] == "linear":
        return _linear_backward(s) if c["back"] else _linear_forward(s)
    return _head_plain(s)


# ------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in double precision; every gradient by automatic differentiation of its definition."""
    s = prepare(case, seed)
    c = s["case"]
    with torch.enable_grad():
        return {"dropout": _exact_dropout, "linear": _exact_linear, "head": _exact_head}[c["op"]](s, c)


def _kept(s, rows, cols):
    """Factors of the elements: 1 / (1 - p) or 0, the generator written out word by word in runs of rows."""
    p = s["case"]["p"]
    out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    if p == 0.0:
        return out.fill_(1.0)
    mask = (1 << 32) - 1
    seed, offset = (int(v) & ((1 << 64) - 1) for v in s["seed"].tolist())
    for a in range(0, rows, 2048):
        r = torch.arange(a, min(a + 2048, rows), device="cuda")[:, None]
        q = torch.arange((cols + 3) // 4, device="cuda")[None, :]
        c0, c1 = q + 0 * r, r + 0 * q
        c2, c3 = torch.full_like(c0, offset & mask), torch.full_like(c0, offset >> 32)
        for i in range(10):
            k0, k1 = ((seed & mask) + i * 0x9E3779B9) & mask, ((seed >> 32) + i * 0xBB67AE85) & mask
            left, right = 0xD2511F53 * c0, 0xCD9E8D57 * c2
            c0, c1, c2, c3 = ((right >> 32) & mask) ^ c1 ^ k0, right & mask, ((left >> 32) & mask) ^ c3 ^ k1, left & mask
        words = torch.stack((c0, c1, c2, c3), -1).flatten(1)[:, :cols]
        out[a:a + 2048] = (words.double() >= p * 2.0 ** 32).double() / (1.0 - p)
    return out


def _exact_dropout(s, c):
    v = s["x"].double() * _kept(s, c["rows"], c["cols"])
    return {"dx": v} if c["back"] else {"out": v + s["residual"].double() if c["residual"] else v}


def _activation(z, act):
    f = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"),
            "silu": lambda: f.silu(z)}[act]()


def _exact_linear(s, c):
    x, w = s["x"].double(), s["w"].double()
    wt = w.t() if c["by_output"] else w
    if not c["back"]:
        z = x @ wt
        if c["bias"]:
            z = z + s["bias"].double()
        out = _activation(z, c["act"]) * _kept(s, *z.shape)
        if c["residual"]:
            out = out + s["residual"].double()
        return _some({"out": out, "pre": z if c["keep_pre"] else None})
    dz = s["dout"].double() * _kept(s, *s["dout"].shape)
    if c["act"] != "none":
        pre = s["pre"].double().requires_grad_()
        dz = torch.autograd.grad((_activation(pre, c["act"]) * dz).sum(), pre)[0]
    dw = torch.einsum("nm,nk->mk", dz, x) if c["by_output"] else torch.einsum("nk,nm->km", x, dz)
    return _some({"dx": torch.einsum("nm,km->nk", dz, wt), "dw": dw, "dbias": dz.sum(0) if c["bias"] else None})


def _exact_head(s, c):
    w = s["w"].detach().double()
    if c["part"] != "fwd":
        w.requires_grad_()
    loss, lse, dh, dw = [], [], [], None
    for a in range(0, c["rows"], 512):
        label = s["label"][a:a + 512].long()
        live = label >= 0
        h = torch.where(live[:, None], s["h"][a:a + 512].double(), 0.0).requires_grad_()
        z = h @ (w.t() if c["by_output"] else w)
        total = torch.logsumexp(z, 1)
        each = torch.where(live, total - torch.gather(z, 1, label.clamp(min=0)[:, None])[:, 0], 0.0)
        loss.append(each.detach())
        lse.append((total * live).detach())
        if c["part"] != "fwd":
            value = (each * s["weight"][a:a + 512].double()).sum()
            got = torch.autograd.grad(value, (h, w))
            dh.append(got[0])
            dw = got[1] if dw is None else dw + got[1]
        del z, total, each
    out = {} if c["part"] == "bwd" else {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    if c["part"] != "fwd":
        out.update(dh=torch.cat(dh), dw=dw)
    return out
