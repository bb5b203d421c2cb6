"""The training-step operators of this framework, in plain form and through its entry points.

Three operators, each forward and backward, as one training step of a profiled model runs them between its matrix
products (every size is in elements, rows are tokens):

    norm      u = y rstd(y) (w_after + o);  x' = x + alpha g u;  h = x' rstd(x') (w_before + o),
              with rstd(v) = 1 / sqrt(mean(v^2) + eps) and g = gate or tanh(gate), one gate row per `group` rows
    router    softmax over the experts, the k largest, their weights, counts and probability sums per group of rows,
              and the balance loss  coef * mean over groups of  E * sum_e (counts_e / (k n)) (probability sum_e / n)
    distill   T^2 KL(q || p) per row, q = softmax(t / T) over a teacher's K logits, p = softmax(z / T) over the vocabulary

`own = False`: elementary torch operations in 32 bits.  `own = True`: the library's kernels.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5
ALPHA = 0.5           # residual scale of the block norm
COEF = 0.01           # coefficient of the balance loss
LOSS_SCALE = 1024.0   # half precision trains under a loss scale: the gradients that come in carry it
NINF = float("-inf")


# ---------------------------------------------------------------------------------------------------------- cases

def _norm(name, back, rows, cols, dtype, **kw):
    c = dict(name=name, op="norm", back=back, rows=rows, cols=cols, dtype=dtype, wtype=dtype, group=0, gated=True, block=True,
             after=True, before=True, tanh=False, offset=False, pad=0)
    c.update(kw)
    return c


def _router(name, back, rows, experts, k, dtype, **kw):
    c = dict(name=name, op="router", back=back, rows=rows, experts=experts, k=k, dtype=dtype, group=0, masked=0, closed=0, renorm=False, pad=0)
    c.update(kw)
    return c


def _distill(name, part, rows, vocab, k, dtype, **kw):
    c = dict(name=name, op="distill", part=part, rows=rows, vocab=vocab, k=k, dtype=dtype, ttype="fp32", padded=0, temperature=1.0, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # a handful of tokens at one block edge: samples drawn from a model between training steps; latency counts
        _norm("norm fwd, 4 tokens", False, 4, 4096, "bf16", group=4),
        # four sequences of 2,048 tokens at the widest hidden size of the paper-scale jobs, one tanh gate row a sequence
        _norm("norm fwd, 4 sequences", False, 8192, 5120, "bf16", group=2048, tanh=True),
        # an odd width in single precision in rows cut from a wider buffer, no gate: a model under test
        _norm("norm fwd, odd width", False, 1000, 1537, "fp32", gated=False, pad=3),
        # one sequence of 2,048 tokens through the backward pass, a learned vector as the gate, single-precision weights
        _norm("norm bwd, 1 sequence", True, 2048, 1280, "fp16", wtype="fp32", group=2048),
        # a micro-batch of eight sequences through the backward pass, one gate row a sequence
        _norm("norm bwd, 8 sequences", True, 16384, 4096, "bf16", group=2048, offset=True),
        # the router of a small mixture on one short sequence; latency counts
        _router("router fwd, 8 experts", False, 512, 8, 2, "bf16"),
        # 32 sequences over many experts, balanced sequence by sequence, logits in single precision, some padding tokens
        _router("router fwd, 128 experts", False, 65536, 128, 8, "fp32", group=2048, masked=500, renorm=True),
        # an odd number of experts of which some are closed for this step, raw weights, rows cut from a wider buffer
        _router("router bwd, 60 experts", True, 3001, 60, 4, "fp32", group=0, closed=5, masked=11, pad=1),
        # the largest router step: 64 sequences, 256 experts, weights normalised over the chosen eight
        _router("router bwd, 256 experts", True, 131072, 256, 8, "bf16", renorm=True),
        # an evaluation batch of few rows over a vocabulary whose rows start at odd addresses
        _distill("distill fwd, 32 rows", "fwd", 32, 50257, 20, "bf16"),
        # the backward pass alone, when the loss is one term of several
        _distill("distill bwd, 1,000 rows", "bwd", 1000, 32000, 64, "fp16", temperature=2.0, ttype="fp16"),
        # a whole training step of the head: loss and gradient of 2,048 tokens at once, the last ones padding
        _distill("distill step, 2,048 rows", "step", 2048, 128000, 64, "bf16", temperature=2.0, padded=48),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, unit):
    """A size between lo and hi, spread over its logarithm: half the time a multiple of `unit`."""
    n = _log(rng, lo, hi)
    return max(unit, n // unit * unit) if rng.random() < 0.5 else n


def _aside(n):
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    op = rng.choice(["norm", "norm", "router", "distill"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 40)])
    size = 4 if dtype == "fp32" else 2
    if op == "norm":
        back = rng.random() < 0.5
        cols = _aside(_size(rng, 64, 8192, 128))
        rows = _aside(_log(rng, 1, min(32768, (1 << 27) // (size * cols))))
        block = rng.random() < 0.85
        after = block and rng.random() < 0.8
        before = not block or rng.random() < 0.85
        gated = block and rng.random() < 0.75
        group = rng.choice([rows, max(1, rows // rng.randint(2, 8)), _log(rng, 1, rows)])
        c = _norm("", back, rows, cols, dtype, wtype=rng.choice([dtype, "fp32"]), group=group if gated else 0, gated=gated, block=block,
                  after=after, before=before, tanh=gated and rng.random() < 0.4, offset=rng.random() < 0.3, pad=pad)
    elif op == "router":
        experts = _aside(_size(rng, 4, 512, 8))
        rows = _aside(_log(rng, 1, min(131072, (1 << 25) // experts)))
        k = rng.randint(1, min(8, experts))
        c = _router("", rng.random() < 0.5, rows, experts, k, dtype, group=rng.choice([0, 0, _log(rng, 1, rows)]),
                    masked=rng.choice([0, rng.randint(0, rows // 4)]), closed=rng.choice([0, rng.randint(0, experts - 1)]),
                    renorm=rng.random() < 0.5, pad=pad)
    else:
        vocab = _aside(_size(rng, 1000, 150000, 64))
        rows = _aside(_log(rng, 1, min(4096, (1 << 28) // (size * vocab))))
        c = _distill("", rng.choice(["fwd", "bwd", "step"]), rows, vocab, _log(rng, 1, 128), dtype, ttype=rng.choice(["fp32", dtype]),
                     padded=rng.choice([0, rng.randint(0, rows // 3)]), temperature=rng.choice([1.0, 2.0, round(rng.uniform(0.5, 4.0), 3)]), pad=pad)
    del c["name"]
    return c


def _groups(c):
    g = c["group"] or c["rows"]
    return g, -(-c["rows"] // g)


def work(case):
    c = case
    b = {"bf16": 2, "fp16": 2, "fp32": 4}
    e, n = b[c["dtype"]], c["rows"]
    if c["op"] == "norm":
        d, (_, ng) = c["cols"], _groups(c)
        blk, bef, aft, gat = c["block"], c["before"], c["after"], c["gated"]
        weights = (aft + bef) * d * b[c["wtype"]]
        if not c["back"]:
            # x, y -> x', h, rstd
            return {"bytes": n * d * e * (1 + 2 * blk + bef) + gat * ng * d * e + weights + 8 * n, "flops": n * d * (4 * aft + 3 * blk + 4 * bef)}
        # dx', (x', dh), y -> dx, dy, dgate and the gradients of the weights
        return {"bytes": n * d * e * (2 + 2 * bef + (aft or gat) * blk + blk) + 2 * gat * ng * d * e + weights + (aft + bef) * d * 4 + 8 * n,
                "flops": n * d * (10 * aft + 4 * blk + 10 * bef)}
    if c["op"] == "router":
        x, k, (_, ng) = c["experts"], c["k"], _groups(c)
        if not c["back"]:
            return {"bytes": n * x * e + n + 8 * n * k + 8 * ng * x + 4 * ng + 4, "flops": n * x * (5 + k)}
        return {"bytes": 2 * n * x * e + (8 if not c["renorm"] else 12) * n * k + 4 * ng * x + 4 * ng + 4, "flops": n * x * 9}
    v, live = c["vocab"], n - c["padded"]
    teacher = n * c["k"] * (4 + b[c["ttype"]])
    if c["part"] == "fwd":
        return {"bytes": live * v * e + teacher + 8 * n, "flops": live * v * 4}
    if c["part"] == "bwd":
        return {"bytes": (live + n) * v * e + teacher + 8 * n, "flops": live * v * 4}
    return {"bytes": (live + n) * v * e + teacher + 12 * n, "flops": live * v * 8}


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

    def normal(rows, cols, scale=1.0, shift=0.0, dtype=t, pad=pad):
        v = _rows(rows, cols, pad, dtype)
        v.copy_(torch.randn(rows, cols, generator=g, device="cuda").mul_(scale).add_(shift))
        return v

    if c["op"] == "norm":
        d, (_, ng) = c["cols"], _groups(c)
        w = TYPES[c["wtype"]]
        off = 0.0 if c["offset"] else 1.0
        vector = lambda: torch.empty(d, dtype=w, device="cuda").copy_(torch.randn(d, generator=g, device="cuda").mul_(0.1).add_(off))  # noqa: E731
        # a residual stream: a few channels are much larger than the rest
        x = normal(n, d, 1.5)
        x[:, :: max(1, d // 7)] *= 8
        s["x"] = x
        s["y"] = normal(n, d, 0.4) if c["block"] else None
        s["w_after"] = vector() if c["after"] else None
        s["w_before"] = vector() if c["before"] else None
        s["gate"] = normal(ng, d, 0.5, 0.2, pad=0) if c["gated"] else None
        s["rstd"] = torch.zeros(n, 2, dtype=torch.float32, device="cuda")
        if c["back"]:
            if c["after"]:
                s["rstd"][:, 0] = (s["y"].float().square().mean(1) + EPS).rsqrt()
            if c["before"]:
                s["rstd"][:, 1] = (x.float().square().mean(1) + EPS).rsqrt()
            s["dx_out"] = normal(n, d, 0.02)
            s["dh"] = normal(n, d, 0.05) if c["before"] else None
            s["out"] = {"dx": _rows(n, d, pad, t), "dy": _rows(n, d, pad, t) if c["block"] else None,
                        "dw_after": torch.empty(d, dtype=torch.float32, device="cuda") if c["after"] else None,
                        "dgate": torch.empty_like(s["gate"]) if c["gated"] else None,
                        "dw_before": torch.empty(d, dtype=torch.float32, device="cuda") if c["before"] else None}
        else:
            s["out"] = {"x_out": _rows(n, d, pad, t) if c["block"] else None, "h": _rows(n, d, pad, t) if c["before"] else None,
                        "rstd": s["rstd"]}
    elif c["op"] == "router":
        x, k, (_, ng) = c["experts"], c["k"], _groups(c)
        # some experts are liked more than others; equal logits are common in 16 bits
        z = normal(n, x, 1.2)
        z += torch.randn(x, generator=g, device="cuda").mul_(0.7).to(t)
        if c["closed"]:
            z[:, torch.randperm(x, generator=g, device="cuda")[: c["closed"]]] = NINF
        s["logits"] = z
        s["mask"] = None
        if c["masked"]:
            s["mask"] = torch.ones(n, dtype=torch.uint8, device="cuda")
            at = torch.randperm(n, generator=g, device="cuda")[: c["masked"]]
            s["mask"][at] = 0
            z[at] = float("nan")                     # what stands in a padding row is nobody's business
        i32 = dict(dtype=torch.int32, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        if c["back"]:
            got = _router_forward(s)
            for key in ("index", "weight", "counts", "valid"):
                s[key] = got[key]
            s["dloss"] = torch.full((1,), scale, **f32)
            s["dweight"] = torch.randn(n, k, generator=g, device="cuda").mul_(0.01 * scale)
            s["out"] = {"dlogits": _rows(n, x, pad, t)}
        else:
            s["out"] = {"index": torch.empty(n, k, **i32), "weight": torch.empty(n, k, **f32), "counts": torch.empty(ng, x, **i32),
                        "prob_sum": torch.empty(ng, x, **f32), "valid": torch.empty(ng, **i32), "loss": torch.empty(1, **f32)}
    else:
        v, k = c["vocab"], min(c["k"], c["vocab"])
        c["k"] = k
        live = n - c["padded"]
        s["z"] = z = normal(n, v, 2.0)
        # the teacher's entries: distinct places, largest logit first; the student likes them as well
        step = torch.randint(1, max(2, v // max(k, 1)), (n, 1), generator=g, device="cuda")
        idx = (torch.randint(0, v, (n, 1), generator=g, device="cuda") + step * torch.arange(k, device="cuda")) % v
        tl = torch.randn(n, k, generator=g, device="cuda").mul_(2.0).add_(12.0).sort(1, descending=True)[0]
        z.scatter_(1, idx, (tl + torch.randn(n, k, generator=g, device="cuda")).to(t))
        # some rows have fewer than K entries (the first stays), padding rows have none
        short = torch.rand(n, k, generator=g, device="cuda") < 0.05
        short[:, 0] = False
        short[live:] = True
        s["index"] = torch.where(short, -1, idx).to(torch.int32)
        s["teacher"] = tl.to(TYPES[c["ttype"]])
        s["weight"] = torch.rand(n, generator=g, device="cuda").add_(0.5) * (scale / n)
        f32 = dict(dtype=torch.float32, device="cuda")
        s["lse"] = torch.zeros(n, **f32)
        if c["part"] == "bwd":
            for a in range(0, n, 256):
                s["lse"][a:a + 256] = torch.logsumexp(z[a:a + 256].float() / c["temperature"], 1)
            s["lse"][live:] = 0
            s["out"] = {"dz": _rows(n, v, pad, t)}
        else:
            s["out"] = {"loss": torch.empty(n, **f32), "lse": s["lse"]}
            if c["part"] == "step":
                s["out"]["dz"] = _rows(n, v, pad, t)
    return s


# ---------------------------------------------------------------------------------------------------- plain forms

def _spread(gate, c):
    g, _ = _groups(c)
    return gate.repeat_interleave(g, 0)[: c["rows"]]


def _some(d):
    return {k: v for k, v in d.items() if v is not None}


def _norm_forward(s):
    c = s["case"]
    o = 1.0 if c["offset"] else 0.0
    x = s["x"].float()
    rstd = torch.zeros(c["rows"], 2, dtype=torch.float32, device="cuda")
    out = {"x_out": None, "h": None, "rstd": rstd}
    if c["block"]:
        u = s["y"].float()
        if c["after"]:
            rstd[:, 0] = (u.square().mean(1) + EPS).rsqrt()
            u = u * rstd[:, :1] * (s["w_after"].float() + o)
        if c["gated"]:
            gate = s["gate"].float()
            u = u * _spread(gate.tanh() if c["tanh"] else gate, c)
        x = x + ALPHA * u
        out["x_out"] = x.to(TYPES[c["dtype"]])
    if c["before"]:
        rstd[:, 1] = (x.square().mean(1) + EPS).rsqrt()
        out["h"] = (x * rstd[:, 1:] * (s["w_before"].float() + o)).to(TYPES[c["dtype"]])
    return _some(out)


def _norm_backward(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    o = 1.0 if c["offset"] else 0.0
    out = {}
    grad = s["dx_out"].float()
    if c["before"]:
        hat = s["x"].float() * s["rstd"][:, 1:]
        dh = s["dh"].float()
        out["dw_before"] = (dh * hat).sum(0)
        dh = dh * (s["w_before"].float() + o)
        grad = grad + s["rstd"][:, 1:] * (dh - hat * (dh * hat).mean(1, keepdim=True))
    out["dx"] = grad.to(t)
    if c["block"]:
        y = s["y"].float()
        hat = y * s["rstd"][:, :1] if c["after"] else y
        w = s["w_after"].float() + o if c["after"] else 1.0
        du = ALPHA * grad
        if c["gated"]:
            gate = s["gate"].float()
            size, ng = _groups(c)
            dg = du * hat * w
            dg = torch.nn.functional.pad(dg, (0, 0, 0, ng * size - c["rows"])).view(ng, size, -1).sum(1)
            if c["tanh"]:
                gate = gate.tanh()
                dg = dg * (1 - gate * gate)
            out["dgate"] = dg.to(t)
            du = du * _spread(gate, c)
        if c["after"]:
            out["dw_after"] = (du * hat).sum(0)
            du = du * w
            du = s["rstd"][:, :1] * (du - hat * (du * hat).mean(1, keepdim=True))
        out["dy"] = du.to(t)
    return out


def _router_forward(s):
    c = s["case"]
    n, x, k = c["rows"], c["experts"], c["k"]
    size, ng = _groups(c)
    z = s["logits"].float()
    if s["mask"] is not None:
        z = torch.where(s["mask"][:, None] != 0, z, NINF)
    top = z.max(1, keepdim=True)[0]
    live = top > NINF
    p = torch.where(live, (z - torch.where(live, top, 0.0)).exp(), 0.0)
    p = torch.where(live, p / p.sum(1, keepdim=True), 0.0)
    value, index = z.sort(dim=1, descending=True, stable=True)
    index = index[:, :k]
    chosen = value[:, :k] > NINF
    weight = torch.where(chosen, p.gather(1, index), 0.0)
    if c["renorm"]:
        weight = torch.where(live, weight / weight.sum(1, keepdim=True), 0.0)
    at = torch.arange(n, device="cuda")[:, None] // size * x + index
    counts = torch.zeros(ng * x, dtype=torch.int32, device="cuda")
    counts.scatter_add_(0, at.reshape(-1), chosen.reshape(-1).to(torch.int32))
    counts = counts.view(ng, x)
    fill = ng * size - n
    prob_sum = torch.nn.functional.pad(p, (0, 0, 0, fill)).view(ng, size, x).sum(1)
    valid = torch.nn.functional.pad(live[:, 0].to(torch.int32), (0, fill)).view(ng, size).sum(1, dtype=torch.int32)
    m = valid.clamp(min=1).float()
    each = (counts.float() * prob_sum).sum(1) * x / (k * m * m)
    loss = COEF * each.sum() / (valid > 0).sum().clamp(min=1).float()
    return {"index": torch.where(chosen, index, -1).to(torch.int32), "weight": weight, "counts": counts, "prob_sum": prob_sum,
            "valid": valid, "loss": loss.view(1)}


def _router_backward(s):
    c = s["case"]
    size, ng = _groups(c)
    x, k = c["experts"], c["k"]
    live = s["index"][:, :1] >= 0
    z = torch.where(live, s["logits"].float(), 0.0)
    p = (z - z.max(1, keepdim=True)[0]).exp()
    p = p / p.sum(1, keepdim=True)
    m = s["valid"].clamp(min=1).float()[:, None]
    pull = s["dloss"] * COEF * x / (k * m * m * (s["valid"] > 0).sum().clamp(min=1).float()) * s["counts"].float()
    dp = pull.repeat_interleave(size, 0)[: c["rows"]]
    chosen = s["index"] >= 0
    at = s["index"].clamp(min=0).long()
    dw = torch.where(chosen, s["dweight"], 0.0)
    if not c["renorm"]:
        dp = dp.scatter_add(1, at, dw)
    dz = p * (dp - (p * dp).sum(1, keepdim=True))
    if c["renorm"]:
        dz = dz.scatter_add(1, at, s["weight"] * (dw - (s["weight"] * dw).sum(1, keepdim=True)))
    return {"dlogits": torch.where(live, dz, 0.0).to(TYPES[c["dtype"]])}


def _teacher(s):
    """q and log q over the teacher's entries (0 and 0 where there is none), and whether there is one."""
    there = s["index"] >= 0
    t = torch.where(there, s["teacher"].float() / s["case"]["temperature"], NINF)
    top = t.max(1, keepdim=True)[0]
    live = top > NINF
    t = t - torch.where(live, top, 0.0)
    total = t.exp().sum(1, keepdim=True)
    log_q = torch.where(there, t - torch.where(live, total, 1.0).log(), 0.0)
    return torch.where(there, log_q.exp(), 0.0), log_q, live


def _distill_forward(s):
    c = s["case"]
    T = c["temperature"]
    q, log_q, live = _teacher(s)
    z = torch.where(live, s["z"].float(), 0.0) / T
    top = z.max(1, keepdim=True)[0]
    rest = (z - top).exp().sum(1, keepdim=True).log()
    log_p = z.gather(1, s["index"].clamp(min=0).long()) - top - rest
    loss = torch.where(live, T * T * (q * (log_q - log_p)).sum(1, keepdim=True), 0.0)
    return {"loss": loss[:, 0], "lse": torch.where(live, top + rest, 0.0)[:, 0]}


def _distill_backward(s, lse):
    c = s["case"]
    T = c["temperature"]
    q, _, live = _teacher(s)
    p = (torch.where(live, s["z"].float(), 0.0) / T - lse[:, None]).exp()
    p = p.scatter_add(1, s["index"].clamp(min=0).long(), -q)
    return {"dz": torch.where(live, s["weight"][:, None] * T * p, 0.0).to(TYPES[c["dtype"]])}


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
        o = s["out"]
        if c["op"] == "norm":
            s["plan"] = binding.block_norm(
                c["rows"], c["cols"], TYPES[c["dtype"]], TYPES[c["wtype"]], eps=EPS, alpha=ALPHA, group_rows=_groups(c)[0], norm_after=c["after"],
                norm_before=c["before"], unit_offset=c["offset"], tanh_gate=c["tanh"], ld=c["cols"] + c["pad"])
        elif c["op"] == "router":
            s["plan"] = binding.router(
                c["rows"], c["experts"], c["k"], TYPES[c["dtype"]], group_rows=_groups(c)[0], coef=COEF, renorm=c["renorm"], ld=c["experts"] + c["pad"])
        else:
            s["plan"] = binding.distill(
                c["rows"], c["vocab"], c["k"], TYPES[c["dtype"]], TYPES[c["ttype"]], temperature=c["temperature"], ld=c["vocab"] + c["pad"])
        s["result"] = _some(o)
    return s["plan"]


def run(state):
    s, c = state, state["case"]
    if own:
        ctx, plan, o = _ctx(), _plan(s), s["out"]
        if c["op"] == "norm":
            if c["back"]:
                ctx.block_norm_backward(plan, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], s["rstd"], s["dx_out"], s["dh"],
                                        o["dx"], o["dy"], o["dw_after"], o["dgate"], o["dw_before"])
            else:
                ctx.block_norm_forward(plan, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], o["x_out"], o["h"], o["rstd"])
        elif c["op"] == "router":
            if c["back"]:
                ctx.router_backward(plan, s["logits"], s["index"], s["weight"], s["counts"], s["valid"], s["dloss"], s["dweight"], o["dlogits"])
            else:
                ctx.router_forward(plan, s["logits"], s["mask"], o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
        elif c["part"] == "fwd":
            ctx.distill_forward(plan, s["z"], s["index"], s["teacher"], o["loss"], o["lse"])
        elif c["part"] == "bwd":
            ctx.distill_backward(plan, s["z"], s["index"], s["teacher"], s["lse"], s["weight"], o["dz"])
        else:
            ctx.distill_step(plan, s["z"], s["index"], s["teacher"], s["weight"], o["loss"], o["lse"], o["dz"])
        return s["result"]
    if c["op"] == "norm":
        return _norm_backward(s) if c["back"] else _norm_forward(s)
    if c["op"] == "router":
        return _router_backward(s) if c["back"] else _router_forward(s)
    if c["part"] == "fwd":
        return _distill_forward(s)
    if c["part"] == "bwd":
        return _distill_backward(s, s["lse"])
    got = _distill_forward(s)
    return {**got, **_distill_backward(s, got["lse"])}


# ------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in double precision; every gradient by automatic differentiation of its definition."""
    s = prepare(case, seed)
    c = s["case"]
    with torch.enable_grad():
        if c["op"] == "norm":
            return _exact_norm(s, c)
        if c["op"] == "router":
            return _exact_router(s, c)
        return _exact_distill(s, c)


def _leaf(v):
    return None if v is None else v.detach().double().requires_grad_()


def _grad(value, leaves):
    at = [v for v in leaves.values() if v is not None]
    got = iter(torch.autograd.grad(value, at))
    return {k: next(got) for k, v in leaves.items() if v is not None}


def _rms(v, w, c):
    scale = torch.pow(torch.mean(v * v, dim=-1, keepdim=True) + EPS, -0.5)
    return v * scale * (w + 1.0 if c["offset"] else w), scale[:, 0]


def _exact_norm(s, c):
    row_of = torch.arange(c["rows"], device="cuda") // _groups(c)[0]

    def edge(y, w, gate):
        u, r = _rms(y, w, c) if c["after"] else (y, torch.zeros_like(y[:, 0]))
        if gate is not None:
            u = u * (torch.tanh(gate) if c["tanh"] else gate)[row_of]
        return ALPHA * u, r

    y, wa, gate, wb = _leaf(s["y"]), _leaf(s["w_after"]), _leaf(s["gate"]), _leaf(s["w_before"])
    x = _leaf(s["x"])
    if not c["back"]:
        out, stream, ra = {}, x, torch.zeros_like(x[:, 0])
        if c["block"]:
            add, ra = edge(y, wa, gate)
            stream = x + add
            out["x_out"] = stream.detach()
        h, rb = _rms(stream, wb, c) if c["before"] else (None, torch.zeros_like(ra))
        if c["before"]:
            out["h"] = h.detach()
        return {**out, "rstd": torch.stack([ra, rb], 1).detach()}
    out, total = {}, s["dx_out"].double()
    if c["before"]:
        got = _grad((_rms(x, wb, c)[0] * s["dh"].double()).sum(), {"x": x, "w": wb})
        total = total + got["x"]
        out["dw_before"] = got["w"]
    out["dx"] = total
    if c["block"]:
        got = _grad((edge(y, wa, gate)[0] * total).sum(), {"dy": y, "dw_after": wa, "dgate": gate})
        out.update(got)
    return out


def _exact_router(s, c):
    size, ng = _groups(c)
    n, x, k = c["rows"], c["experts"], c["k"]
    z = s["logits"].detach().double()
    keep = torch.ones(n, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"].bool()
    open_ = (z > NINF) & keep[:, None]
    keep = open_.any(1)
    z = torch.where(keep[:, None], z, torch.zeros_like(z)).requires_grad_()
    p = torch.softmax(z, 1) * keep[:, None]
    order = torch.argsort(torch.where(open_, z, NINF), dim=1, descending=True, stable=True)[:, :k]
    chosen = torch.gather(open_, 1, order)
    weight = torch.gather(p, 1, order) * chosen
    if c["renorm"]:
        weight = weight / torch.where(keep, weight.sum(1), 1.0)[:, None]
    group = torch.arange(n, device="cuda") // size
    hit = torch.zeros(n, x, dtype=torch.float64, device="cuda").scatter_(1, order, chosen.double())
    zero = torch.zeros(ng, x, dtype=torch.float64, device="cuda")
    counts, sums = zero.index_add(0, group, hit), zero.index_add(0, group, p)
    valid = torch.zeros(ng, dtype=torch.float64, device="cuda").index_add(0, group, keep.double())
    some = valid > 0
    f, mean = counts / (k * valid.clamp(min=1))[:, None], sums / valid.clamp(min=1)[:, None]
    loss = COEF * x * (f * mean).sum() / max(1, int(some.sum()))
    if c["back"]:
        value = loss * s["dloss"].double()[0] + (weight * s["dweight"].double()).sum()
        return {"dlogits": torch.nan_to_num(torch.autograd.grad(value, z)[0], nan=0.0) * keep[:, None]}
    return {"index": torch.where(chosen, order, -1).int(), "weight": weight.detach(), "counts": counts.int(), "prob_sum": sums.detach(),
            "valid": valid.int(), "loss": loss.detach().view(1)}


def _exact_distill(s, c):
    n, T = c["rows"], c["temperature"]
    outs = {k: [] for k in ("loss", "lse", "dz")}
    for a in range(0, n, 256):
        idx = s["index"][a:a + 256].long()
        there = idx >= 0
        live = there.any(1)
        z = torch.where(live[:, None], s["z"][a:a + 256].double(), 0.0).requires_grad_()
        t = torch.where(there, s["teacher"][a:a + 256].double(), NINF) / T
        q = torch.softmax(torch.where(live[:, None], t, 0.0), 1) * there
        lse = torch.logsumexp(z / T, 1)
        log_p = torch.gather(z / T, 1, idx.clamp(min=0)) - lse[:, None]
        loss = T * T * (torch.xlogy(q, q) - q * log_p).sum(1) * live
        outs["loss"].append(loss.detach())
        outs["lse"].append((lse * live).detach())
        if c["part"] != "fwd":
            weight = s["weight"][a:a + 256].double()
            outs["dz"].append(torch.autograd.grad((loss * weight).sum(), z)[0])
    names = {"fwd": ("loss", "lse"), "bwd": ("dz",), "step": ("loss", "lse", "dz")}[c["part"]]
    return {k: torch.cat(outs[k]) for k in names}
