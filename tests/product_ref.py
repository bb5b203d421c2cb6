"""Linear layer, dropout and the head's cross entropy in double precision on the CPU, written out from their definitions,
each with the size of the terms that its sums are made of (what the tests' tolerances are multiples of)."""
import math

import numpy as np
import torch

MASK = (1 << 32) - 1


def philox(counter, key):
    """Philox4x32-10 of one counter, in whole numbers (Salmon et al., SC 2011)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def keep(seed, rows, cols, p, first_row=0):
    """[rows, cols]: 1 / (1 - p) where the element is kept, else 0."""
    if p == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    p = float(np.float32(p))
    s, o = (int(v) & ((1 << 64) - 1) for v in seed)
    quads = -(-cols // 4)
    u = np.uint64
    c = [np.broadcast_to(np.arange(quads, dtype=u), (rows, quads)), np.broadcast_to(np.arange(first_row, first_row + rows, dtype=u)[:, None], (rows, quads)),
         np.full((rows, quads), o & MASK, u), np.full((rows, quads), o >> 32, u)]
    k = [s & MASK, s >> 32]
    low = u(MASK)
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)          # 32 x 32 bits: no overflow
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    words = np.stack(c, 2).reshape(rows, 4 * quads)[:, :cols]
    return torch.from_numpy((words >= u(int(p * 2.0 ** 32))).astype(np.float64)) / (1.0 - p)


def act(z, name):
    f = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "gelu": lambda: 0.5 * z * torch.special.erfc(-z * math.sqrt(0.5)),
            "gelu_tanh": lambda: f.gelu(z, approximate="tanh"), "silu": lambda: f.silu(z)}[name]()


DEVICE = "cpu"           # large products are worked out on the GPU, by torch in double precision


def d64(t):
    return None if t is None else t.detach().double().to(DEVICE)


def linear_forward(x, w, bias=None, residual=None, *, activation="none", by_output=False, seed=None, p=0.0):
    """-> out, pre, term sizes of both"""
    x, w, bias, residual = map(d64, (x, w, bias, residual))
    w = w.t() if by_output else w
    z, size = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, size = z + bias, size + bias.abs()
    factor = keep(seed, *z.shape, p).to(z.device)
    out = act(z, activation) * factor
    out = torch.where(factor == 0, 0.0, out)
    size_out = 1.2 * size * factor                     # (no activation's slope exceeds 1.2)
    if residual is not None:
        out, size_out = out + residual, size_out + residual.abs()
    return out, z, size_out, size


def linear_backward(x, w, pre, dout, *, activation="none", by_output=False, seed=None, p=0.0):
    """-> {name: (gradient, term size)}"""
    x, w, pre, dout = map(d64, (x, w, pre, dout))
    factor = keep(seed, *dout.shape, p).to(dout.device)
    dz = torch.where(factor == 0, 0.0, dout * factor)
    if activation != "none":
        z = pre.clone().requires_grad_()
        dz = dz * torch.autograd.grad(act(z, activation).sum(), z)[0]
    size = 1.2 * (dout * factor).abs() if activation != "none" else dz.abs()
    got = {"dbias": (dz.sum(0), size.sum(0))}
    if x is not None and w is not None:
        wt = w if by_output else w.t()
        dw, size_w = x.t() @ dz, x.t().abs() @ size
        got["dw"] = (dw.t(), size_w.t()) if by_output else (dw, size_w)
        got["dx"] = dz @ wt, size @ wt.abs()
    return got


def head(h, w, label, dloss=None, *, by_output=False, lse=None):
    """-> {name: (value, term size)}; rows without a label are left out whatever they hold"""
    h, w, dloss, lse = map(d64, (h, w, dloss, lse))
    w = w.t() if by_output else w                      # [hidden, vocab]
    label = label.long().to(h.device)
    live = (label >= 0) & (label < w.shape[1])
    h = torch.where(live[:, None], h, 0.0)
    z, size = h @ w, h.abs() @ w.abs()
    at = label.clamp(0, w.shape[1] - 1)[:, None]
    total = torch.logsumexp(z, 1)
    worst = size.max(1)[0]
    got = {"loss": (torch.where(live, total - z.gather(1, at)[:, 0], 0.0), worst), "lse": (torch.where(live, total, 0.0), worst)}
    g = torch.ones(len(h), dtype=torch.float64, device=h.device) if dloss is None else dloss
    g = torch.where(live, g, 0.0)
    p = torch.exp(z - (total if lse is None else lse)[:, None])
    hit = torch.zeros_like(z).scatter_(1, at, 1.0)
    dz = torch.where(live[:, None], g[:, None] * (p - hit), 0.0)
    # an exponential is off by what its argument is off by
    size_dz = torch.where(live[:, None], g.abs()[:, None] * (p * (1 + size + worst[:, None]) + hit), 0.0)
    got["dh"] = dz @ w.t(), dz.abs() @ w.t().abs(), size_dz @ w.t().abs()
    dw = h.t() @ dz, h.t().abs() @ dz.abs(), h.t().abs() @ size_dz
    got["dw"] = tuple(v.t() for v in dw) if by_output else dw
    return got
