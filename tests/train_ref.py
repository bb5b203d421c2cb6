"""The training-step operators in double precision, written out from their definitions on the CPU, each with the size
of the terms that its single-precision sums are made of (what the tests' tolerances are multiples of)."""
import torch

NINF = float("-inf")


def rows_of(v, group_rows, rows):
    return v.repeat_interleave(group_rows, 0)[:rows]


def norm_forward(x, y=None, w_after=None, gate=None, w_before=None, *, after=True, before=True, offset=False, tanh=False,
                 eps=1e-5, alpha=1.0, group_rows=1):
    """-> x_out, h, rstd [rows, 2], and the term sizes of x_out and h"""
    f = lambda t: None if t is None else t.detach().double().cpu()  # noqa: E731
    x, y, w_after, gate, w_before = map(f, (x, y, w_after, gate, w_before))
    o = 1.0 if offset else 0.0
    rstd = torch.zeros(len(x), 2, dtype=torch.float64)
    size = x.abs()
    if y is not None:
        u = y
        if after:
            rstd[:, 0] = 1 / torch.sqrt((y * y).mean(1) + eps)
            u = u * rstd[:, :1] * (1.0 if w_after is None else w_after + o)
        if gate is not None:
            u = u * rows_of(torch.tanh(gate) if tanh else gate, group_rows, len(x))
        size = x.abs() + (alpha * u).abs()
        x = x + alpha * u
    h = size_h = None
    if before:
        rstd[:, 1] = 1 / torch.sqrt((x * x).mean(1) + eps)
        w = torch.ones(x.shape[1], dtype=torch.float64) if w_before is None else w_before + o
        h, size_h = x * rstd[:, 1:] * w, size * rstd[:, 1:] * w.abs()
    return x, h, rstd, size, size_h


def norm_backward(x_out, y, w_after, gate, w_before, rstd, dx_out, dh, *, after=True, before=True, offset=False, tanh=False,
                  alpha=1.0, group_rows=1):
    """-> {name: (gradient, term size)}"""
    f = lambda t: None if t is None else t.detach().double().cpu()  # noqa: E731
    x_out, y, w_after, gate, w_before, rstd, dx_out, dh = map(f, (x_out, y, w_after, gate, w_before, rstd, dx_out, dh))
    o = 1.0 if offset else 0.0
    got = {}
    rows, cols = (dh if dh is not None else dx_out).shape
    grad = torch.zeros(rows, cols, dtype=torch.float64) if dx_out is None else dx_out
    size = grad.abs()
    if before:
        rb = rstd[:, 1:]
        xh = x_out * rb
        got["dw_before"] = (dh * xh).sum(0), (dh * xh).abs().sum(0)
        e = dh * (1.0 if w_before is None else w_before + o)
        grad = grad + rb * (e - xh * (e * xh).mean(1, keepdim=True))
        size = size + rb * (e.abs() + xh.abs() * (e * xh).abs().mean(1, keepdim=True))
    got["dx"] = grad, size
    if y is not None:
        ra = rstd[:, :1] if after else torch.ones(rows, 1, dtype=torch.float64)
        yh = y * ra
        w = torch.ones(cols, dtype=torch.float64) if w_after is None else w_after + o
        g = torch.ones(rows, cols, dtype=torch.float64)
        if gate is not None:
            slope = 1 - torch.tanh(gate) ** 2 if tanh else torch.ones_like(gate)
            g = rows_of(torch.tanh(gate) if tanh else gate, group_rows, rows)
            groups = torch.arange(rows) // group_rows
            t = alpha * yh * w
            zero = torch.zeros_like(gate)
            got["dgate"] = slope * zero.index_add(0, groups, grad * t), slope * zero.index_add(0, groups, size * t.abs())
        f1 = alpha * g * grad
        sf = (alpha * g).abs() * size
        if after:
            got["dw_after"] = (f1 * yh).sum(0), (sf * yh.abs()).sum(0)
            f1, sf = f1 * w, sf * w.abs()
            got["dy"] = (ra * (f1 - yh * (f1 * yh).mean(1, keepdim=True)),
                         ra * (sf + yh.abs() * (sf * yh.abs()).mean(1, keepdim=True)))
        else:
            got["dy"] = f1, sf
    return got


def router_forward(logits, mask, k, *, group_rows, coef, renorm):
    z = logits.detach().double().cpu()
    rows, experts = z.shape
    keep = torch.ones(rows, dtype=torch.bool) if mask is None else mask.cpu() != 0
    z = torch.where(keep[:, None], z, torch.full_like(z, NINF))
    keep = (z > NINF).any(1)
    p = torch.where(keep[:, None], torch.softmax(torch.where(keep[:, None], z, torch.zeros_like(z)), 1), torch.zeros_like(z))
    index = torch.full((rows, k), -1, dtype=torch.int64)
    for j in range(k):                                   # one maximum after the other; the first among equals
        at = torch.tensor([max(range(experts), key=lambda e: (row[e], -e)) for row in z.tolist()], dtype=torch.int64)
        value = z.gather(1, at[:, None])[:, 0]
        index[:, j] = torch.where(value > NINF, at, -1)
        z = z.scatter(1, at[:, None], NINF)
    chosen = index >= 0
    weight = torch.where(chosen, p.gather(1, index.clamp(min=0)), torch.zeros(1, dtype=torch.float64))
    if renorm:
        weight = weight / torch.where(keep, weight.sum(1), torch.ones(1, dtype=torch.float64))[:, None]
    groups = -(-rows // group_rows)
    counts = torch.zeros(groups, experts, dtype=torch.int64)
    sums = torch.zeros(groups, experts, dtype=torch.float64)
    valid = torch.zeros(groups, dtype=torch.int64)
    total, some = 0.0, 0
    for g in range(groups):
        part = slice(g * group_rows, (g + 1) * group_rows)
        hit = index[part][chosen[part]]
        counts[g] = torch.bincount(hit, minlength=experts)
        sums[g] = p[part].sum(0)
        valid[g] = keep[part].sum()
        n = int(valid[g])
        if n:
            some += 1
            total += experts * float((counts[g] / (k * n) * sums[g] / n).sum())
    return dict(index=index, weight=weight, counts=counts, prob_sum=sums, valid=valid, loss=coef * total / max(some, 1), p=p)


def router_backward(fwd, k, dloss, dweight, *, group_rows, coef, renorm):
    """-> dlogits and its term size, from router_forward's answer"""
    p, index, w = fwd["p"], fwd["index"], fwd["weight"]
    rows, experts = p.shape
    some = max(int((fwd["valid"] > 0).sum()), 1)
    n = fwd["valid"].clamp(min=1).double()[:, None]
    a = rows_of(dloss * coef * experts * fwd["counts"].double() / (some * k * n * n), group_rows, rows)
    d = torch.zeros(rows, k, dtype=torch.float64) if dweight is None else torch.where(index >= 0, dweight.double().cpu(), 0.0)
    at = index.clamp(min=0)
    wd, swd = (w * d).sum(1, keepdim=True), (w * d).abs().sum(1, keepdim=True)
    dp = a if renorm else a.scatter_add(1, at, d)
    sp = a.abs() if renorm else a.abs().scatter_add(1, at, d.abs())
    dz = p * (dp - (p * dp).sum(1, keepdim=True))
    size = p * (sp + (p * sp).sum(1, keepdim=True))
    if renorm:
        dz = dz.scatter_add(1, at, w * (d - wd))
        size = size.scatter_add(1, at, w * (d.abs() + swd))
    live = index[:, :1] >= 0
    return torch.where(live, dz, 0.0), torch.where(live, size, 0.0)


def distill(z, index, teacher, temperature, dloss=None):
    """-> loss, lse, dz, and their term sizes"""
    z, teacher, index = z.detach().double().cpu(), teacher.detach().double().cpu(), index.cpu().long()
    rows, vocab = z.shape
    T = temperature
    there = (index >= 0) & (index < vocab) & (teacher > NINF)
    live = there.any(1)
    up = torch.ones(rows, dtype=torch.float64) if dloss is None else dloss.detach().double().cpu()
    loss, lse, s_loss, s_lse = (torch.zeros(rows, dtype=torch.float64) for _ in range(4))
    dz, s_dz = torch.zeros_like(z), torch.zeros_like(z)
    for r in range(rows):
        if not live[r]:
            continue
        i, t = index[r][there[r]], teacher[r][there[r]] / T
        log_q = t - torch.logsumexp(t, 0)
        q = log_q.exp()
        s = z[r] / T
        lse[r] = torch.logsumexp(s, 0)
        log_p = torch.where(z[r] > NINF, s - lse[r], NINF)
        loss[r] = T * T * (q * (log_q - log_p[i]))[q > 0].sum()
        top = s[s > NINF].abs().max() if (s > NINF).any() else 0.0
        s_loss[r] = T * T * (q * (log_q.abs() + torch.where(log_p[i] > NINF, log_p[i].abs(), 0.0) + 1)).sum()
        s_lse[r] = top + 1
        p = log_p.exp()
        grad = p.clone().index_add(0, i, -q)
        size = p.clone().index_add(0, i, q)
        dz[r], s_dz[r] = up[r] * T * grad, up[r].abs() * T * size
    return dict(loss=loss, lse=lse, dz=dz, s_loss=s_loss, s_lse=s_lse, s_dz=s_dz)
