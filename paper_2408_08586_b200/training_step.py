"""One training step of a small model, built from the library's training-step operators.

The scheduler plans with what a profile of a job measured: tau, the forward seconds of a sample, and k_bwd, the backward
pass's multiple of it (rubick_job; the profiling runs of the paper's Section 4.3).  This module is such a step on the GPU
at hand: a block, a mixture of experts and a distillation head, with the block norms, the router with its balance loss
and the distillation loss of ``include/rubick.h`` between them, forward and backward.  The blocks themselves are plain
matrix products by torch (a job's own framework would run its own); everything between them is the library's.

It is a sample of how the operators are used together, not a model: a block here is one product, without attention, and
measure() scales such layers up.  A job's own tau and k_bwd come from a profile of the job itself, and its coefficients
from rubick_fit_models.

    x0 -> norm -> block -> [norm, gate, + alpha, norm] -> router -> experts -> [norm, gate, + alpha, norm] -> head -> loss

DenseStep is the step of a model without experts that learns from labels, with its products, its dropout and its head's
cross entropy by the library too:

    x0 -> dropout -> [norm -> up, gelu -> down, dropout, +] -> norm -> head, cross entropy
"""
import torch

from . import binding as rb

PARAMETERS = ("w_in", "w_block", "w_after1", "gate1", "w_before2", "w_router", "w_expert", "w_after2", "gate2", "w_before3", "w_head")


class TrainingStep:
    """Holds the parameters, the descriptors and the buffers of a step of `tokens` tokens.

    ctx: a binding.Context on the stream that torch works on; seq: tokens that are balanced together and share a gate row;
    teacher: entries per token of the teacher."""

    def __init__(self, ctx, tokens, hidden, vocab, *, seq=None, experts=8, chosen=2, teacher=32, dtype=torch.bfloat16,
                 temperature=2.0, alpha=0.5, coef=0.01, seed=0, device="cuda:0"):
        self.ctx, self.tokens, self.hidden, self.vocab = ctx, int(tokens), int(hidden), int(vocab)
        self.experts, self.chosen, self.dtype, self.coef = int(experts), int(chosen), dtype, float(coef)
        seq = self.tokens if seq is None else int(seq)
        self.groups = -(-self.tokens // seq)
        n, d, v, e, k = self.tokens, self.hidden, self.vocab, self.experts, self.chosen
        g = torch.Generator(device=device).manual_seed(seed)
        draw = lambda *shape, scale=1.0, shift=0.0: torch.randn(*shape, generator=g, device=device).mul_(scale).add_(shift).to(dtype)  # noqa: E731
        self.p = dict(w_in=draw(d, scale=0.1, shift=1.0), w_block=draw(d, d, scale=d ** -0.5), w_after1=draw(d, scale=0.1, shift=1.0),
                      gate1=draw(self.groups, d, scale=0.3, shift=0.5), w_before2=draw(d, scale=0.1, shift=1.0),
                      w_router=draw(d, e, scale=d ** -0.5), w_expert=draw(e, d, d, scale=d ** -0.5), w_after2=draw(d, scale=0.1, shift=1.0),
                      gate2=draw(self.groups, d, scale=0.3, shift=0.5), w_before3=draw(d, scale=0.1, shift=1.0),
                      w_head=draw(d, v, scale=d ** -0.5))
        self.first = rb.block_norm(n, d, dtype, norm_after=False)
        self.edge = rb.block_norm(n, d, dtype, alpha=alpha, group_rows=seq, tanh_gate=True)
        self.route = rb.router(n, e, k, dtype, group_rows=seq, coef=coef, renorm=True)
        self.loss = rb.distill(n, v, teacher, dtype, torch.float32, temperature=temperature)
        rows = lambda *shape: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=device)  # noqa: E731
        i32 = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=device)  # noqa: E731
        self.b = dict(h0=rows(n, d), x1=rows(n, d), h1=rows(n, d), x2=rows(n, d), h2=rows(n, d), r0=f32(n, 2), r1=f32(n, 2), r2=f32(n, 2),
                      index=i32(n, k), weight=f32(n, k), counts=i32(self.groups, e), prob_sum=f32(self.groups, e), valid=i32(self.groups),
                      balance=f32(1), kd=f32(n), lse=f32(n), dz=rows(n, v), dlogits=rows(n, e), dx=rows(n, d), dy=rows(n, d))
        self.g = {name: f32(d) for name in ("w_in", "w_after1", "w_before2", "w_after2", "w_before3")}
        self.g.update(gate1=rows(self.groups, d), gate2=rows(self.groups, d))

    # ---- the experts: every expert's tokens in one product, in the order of (expert, token)

    def _experts_forward(self, h):
        b = self.b
        order = torch.argsort(b["index"].reshape(-1), stable=True)
        self.bounds = [0] + torch.cumsum(b["counts"].sum(0), 0).tolist()
        self.token = order // self.chosen
        self.place = torch.empty_like(order)
        self.place[order] = torch.arange(len(order), device=order.device)
        self.taken = h[self.token]
        self.made = torch.empty_like(self.taken)
        for e in range(self.experts):
            a, z = self.bounds[e], self.bounds[e + 1]
            torch.matmul(self.taken[a:z], self.p["w_expert"][e], out=self.made[a:z])
        made = self.made[self.place].view(self.tokens, self.chosen, self.hidden)
        return (made.float() * b["weight"][..., None]).sum(1).to(self.dtype)

    def _experts_backward(self, dy):
        b = self.b
        dy = dy.float()
        made = self.made[self.place].view(self.tokens, self.chosen, self.hidden)
        dweight = (made.float() * dy[:, None]).sum(-1)
        dmade = (dy[:, None] * b["weight"][..., None]).to(self.dtype).reshape(-1, self.hidden)
        dmade = dmade[torch.argsort(self.place)]
        dtaken = torch.empty_like(dmade)
        self.g["w_expert"] = torch.zeros_like(self.p["w_expert"])
        for e in range(self.experts):
            a, z = self.bounds[e], self.bounds[e + 1]
            torch.matmul(dmade[a:z], self.p["w_expert"][e].t(), out=dtaken[a:z])
            torch.matmul(self.taken[a:z].t(), dmade[a:z], out=self.g["w_expert"][e])
        dh = dtaken[self.place].view(self.tokens, self.chosen, self.hidden).float().sum(1)
        return dh, dweight

    # ---- the step

    def hidden_states(self, x):
        """Everything before the head."""
        c, p, b = self.ctx, self.p, self.b
        self.x0 = x
        c.block_norm_forward(self.first, x, None, None, None, p["w_in"], None, b["h0"], b["r0"])
        self.y1 = b["h0"] @ p["w_block"]
        c.block_norm_forward(self.edge, x, self.y1, p["w_after1"], p["gate1"], p["w_before2"], b["x1"], b["h1"], b["r1"])
        self.logits = b["h1"] @ p["w_router"]
        c.router_forward(self.route, self.logits, None, b["index"], b["weight"], b["counts"], b["prob_sum"], b["valid"], b["balance"])
        self.y2 = self._experts_forward(b["h1"])
        c.block_norm_forward(self.edge, b["x1"], self.y2, p["w_after2"], p["gate2"], p["w_before3"], b["x2"], b["h2"], b["r2"])
        return b["h2"]

    def forward(self, x, index, teacher):
        """-> (distillation loss of every token, balance loss); index, teacher: the teacher's entries [tokens, K]."""
        self.index, self.teacher = index, teacher
        self.z = self.hidden_states(x) @ self.p["w_head"]
        self.ctx.distill_forward(self.loss, self.z, index, teacher, self.b["kd"], self.b["lse"])
        return self.b["kd"], self.b["balance"]

    def backward(self, token_weight=None):
        """Gradients of sum(token_weight * distillation loss) + balance loss -> {parameter: gradient}, and of x under "x"."""
        self.ctx.distill_backward(self.loss, self.z, self.index, self.teacher, self.b["lse"], token_weight, self.b["dz"])
        return self._backward_from(self.b["dz"])

    def step(self, x, index, teacher, token_weight=None):
        """Forward and backward pass with the head's loss and gradient in one kernel -> (losses, balance loss, gradients)."""
        z = self.hidden_states(x) @ self.p["w_head"]
        self.ctx.distill_step(self.loss, z, index, teacher, token_weight, self.b["kd"], self.b["lse"], z)      # over the logits
        return self.b["kd"], self.b["balance"], self._backward_from(z)

    def _backward_from(self, dz):
        c, p, b, g = self.ctx, self.p, self.b, self.g
        g["w_head"] = b["h2"].t() @ dz
        dh2 = dz @ p["w_head"].t()
        c.block_norm_backward(self.edge, b["x2"], self.y2, p["w_after2"], p["gate2"], p["w_before3"], b["r2"], None, dh2, b["dx"], b["dy"],
                              g["w_after2"], g["gate2"], g["w_before3"])
        dh1, dweight = self._experts_backward(b["dy"])
        c.router_backward(self.route, self.logits, b["index"], b["weight"], b["counts"], b["valid"], None, dweight, b["dlogits"])
        g["w_router"] = b["h1"].t() @ b["dlogits"]
        dh1 = (dh1 + (b["dlogits"] @ p["w_router"].t()).float()).to(self.dtype)
        c.block_norm_backward(self.edge, b["x1"], self.y1, p["w_after1"], p["gate1"], p["w_before2"], b["r1"], b["dx"], dh1, b["dx"], b["dy"],
                              g["w_after1"], g["gate1"], g["w_before2"])
        g["w_block"] = b["h0"].t() @ b["dy"]
        dh0 = b["dy"] @ p["w_block"].t()
        c.block_norm_backward(self.first, self.x0, None, None, None, p["w_in"], b["r0"], b["dx"], dh0, b["dx"], None, None, None, g["w_in"])
        return {**{name: g[name] for name in PARAMETERS}, "x": b["dx"]}


DENSE_PARAMETERS = ("w_in", "w_up", "b_up", "w_down", "b_down", "w_out", "w_head")


class DenseStep:
    """Holds the parameters, the descriptors and the buffers of a step of `tokens` tokens in a 16-bit type.

    inner: features between the block's products; drop: probability of both dropouts; tied: the head's weight has a row per
    token of the vocabulary, as an embedding has.  The masks of a step come from self.seed, on the device: advance() draws new
    ones for the next step, also inside of a captured graph."""

    def __init__(self, ctx, tokens, hidden, vocab, *, inner=None, drop=0.1, tied=True, dtype=torch.bfloat16, seed=0, device="cuda:0"):
        self.ctx, self.tokens, self.hidden, self.vocab, self.dtype = ctx, int(tokens), int(hidden), int(vocab), dtype
        self.inner = 4 * self.hidden if inner is None else int(inner)
        n, d, m, v = self.tokens, self.hidden, self.inner, self.vocab
        g = torch.Generator(device=device).manual_seed(seed)
        draw = lambda *shape, scale=1.0, shift=0.0: torch.randn(*shape, generator=g, device=device).mul_(scale).add_(shift).to(dtype)  # noqa: E731
        self.p = dict(w_in=draw(d, scale=0.1, shift=1.0), w_up=draw(d, m, scale=d ** -0.5), b_up=draw(m, scale=0.1), w_down=draw(m, d, scale=m ** -0.5),
                      b_down=draw(d, scale=0.1), w_out=draw(d, scale=0.1, shift=1.0),
                      w_head=draw(v, d, scale=d ** -0.5) if tied else draw(d, v, scale=d ** -0.5))
        self.enter = rb.dropout(n, d, dtype, p=drop)
        self.norm = rb.block_norm(n, d, dtype, norm_after=False)
        self.up = rb.linear(n, d, m, dtype, activation="gelu")
        self.down = rb.linear(n, m, d, dtype, p=drop)
        self.loss = rb.head_loss(n, d, v, dtype, by_output=tied)
        self.seed = torch.tensor([[seed, 0], [seed, 1]], dtype=torch.int64, device=device)
        rows = lambda *shape: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=device)  # noqa: E731
        self.b = dict(x=rows(n, d), h0=rows(n, d), r0=f32(n, 2), pre=rows(n, m), a=rows(n, m), x1=rows(n, d), h1=rows(n, d), r1=f32(n, 2), nll=f32(n), lse=f32(n),
                      dh=rows(n, d), dx=rows(n, d), da=rows(n, m))
        self.g = {name: f32(d) if name in ("w_in", "w_out", "b_down") else f32(m) if name == "b_up" else torch.empty_like(self.p[name]) for name in DENSE_PARAMETERS}

    def advance(self):
        """Other masks from here on."""
        self.seed[:, 1] += 2

    def hidden_states(self, x):
        """Everything before the head."""
        c, p, b = self.ctx, self.p, self.b
        c.dropout_forward(self.enter, self.seed[0], x, None, b["x"])
        c.block_norm_forward(self.norm, b["x"], None, None, None, p["w_in"], None, b["h0"], b["r0"])
        c.linear_forward(self.up, b["h0"], p["w_up"], p["b_up"], None, None, b["pre"], b["a"])
        c.linear_forward(self.down, b["a"], p["w_down"], p["b_down"], b["x"], self.seed[1], None, b["x1"])
        c.block_norm_forward(self.norm, b["x1"], None, None, None, p["w_out"], None, b["h1"], b["r1"])
        return b["h1"]

    def forward(self, x, label):
        """-> cross entropy of every token; label: int32 [tokens], tokens with a negative label are left out."""
        self.label = label
        self.ctx.head_loss_forward(self.loss, self.hidden_states(x), self.p["w_head"], label, self.b["nll"], self.b["lse"])
        return self.b["nll"]

    def backward(self, token_weight=None):
        """Gradients of sum(token_weight * cross entropy) -> {parameter: gradient}, and of x under "x"."""
        self.ctx.head_loss_backward(self.loss, self.b["h1"], self.p["w_head"], self.label, self.b["lse"], token_weight, self.b["dh"], self.g["w_head"])
        return self._backward_from_head()

    def step(self, x, label, token_weight=None):
        """Forward and backward pass with the head's loss and gradients in one call -> (losses, gradients)."""
        self.ctx.head_loss_step(self.loss, self.hidden_states(x), self.p["w_head"], label, token_weight, self.b["nll"], None, self.b["dh"], self.g["w_head"])
        return self.b["nll"], self._backward_from_head()

    def _backward_from_head(self):
        c, p, b, g = self.ctx, self.p, self.b, self.g
        c.block_norm_backward(self.norm, b["x1"], None, None, None, p["w_out"], b["r1"], None, b["dh"], b["dx"], None, None, None, g["w_out"])
        c.linear_backward(self.down, b["a"], p["w_down"], None, self.seed[1], b["dx"], b["da"], g["w_down"], g["b_down"])
        c.linear_backward(self.up, b["h0"], p["w_up"], b["pre"], None, b["da"], b["dh"], g["w_up"], g["b_up"])
        c.block_norm_backward(self.norm, b["x"], None, None, None, p["w_in"], b["r0"], b["dx"], b["dh"], b["dx"], None, None, None, g["w_in"])
        c.dropout_backward(self.enter, self.seed[0], b["dx"], b["dx"])
        return {**g, "x": b["dx"]}


def draw_labels(step, seed=0):
    """(x, labels) for a DenseStep: a random stream and random tokens."""
    g = torch.Generator(device=step.p["w_in"].device).manual_seed(seed)
    x = torch.randn(step.tokens, step.hidden, generator=g, device=step.p["w_in"].device).to(step.dtype)
    return x, torch.randint(0, step.vocab, (step.tokens,), generator=g, device=x.device).to(torch.int32)


def draw_batch(step, seed=0):
    """(x, teacher indices, teacher logits) for a step: a random residual stream, distinct entries, largest first."""
    g = torch.Generator(device=step.p["w_in"].device).manual_seed(seed)
    n, k, device = step.tokens, step.loss.k, step.p["w_in"].device
    x = torch.randn(n, step.hidden, generator=g, device=device).to(step.dtype)
    stride = max(step.vocab // k, 1)
    index = (torch.randint(0, step.vocab, (n, 1), generator=g, device=device) + stride * torch.arange(k, device=device)) % step.vocab
    teacher = torch.randn(n, k, generator=g, device=device).mul_(2).sort(1, descending=True)[0]
    return x, index.to(torch.int32), teacher


def measure(step, layers, seq, repeats=10):
    """Times a step (either kind) on the GPU and scales it to a model of `layers` such layers and one head.
    -> dict(tau, k_bwd): forward seconds per sample of `seq` tokens, backward / forward, as rubick_job takes them."""
    batch = draw_labels(step) if isinstance(step, DenseStep) else draw_batch(step)
    x = batch[0]
    samples = step.tokens / seq

    def seconds(f):
        for _ in range(3):
            f()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        begin.record()
        for _ in range(repeats):
            f()
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end) / 1e3 / repeats

    body = seconds(lambda: step.hidden_states(x))
    forward = seconds(lambda: step.forward(*batch))
    both = seconds(lambda: (step.forward(*batch), step.backward()))
    back = max(both - forward, 0.0)
    head_share = max(forward - body, 0.0) / forward
    whole = body * layers + max(forward - body, 0.0)
    whole_back = back * (1 - head_share) * layers + back * head_share
    return dict(tau=whole / samples, k_bwd=whole_back / whole)


def main():
    """Profiles three model sizes on this GPU and plans a cluster of them."""
    import numpy as np

    from . import workloads
    cfg = workloads.make("paper-scale", J=3)
    plans, _ = rb.enumerate_plans(cfg["g_levels"])
    ctx = rb.Context(cfg["env"], stream=torch.cuda.current_stream().cuda_stream)
    ctx.set_space(plans, cfg["g_levels"], cfg["c_levels"], cfg["m_levels"])
    jobs = cfg["jobs"]
    for j, (hidden, layers, seq) in enumerate([(768, 12, 512), (1280, 24, 1024), (2048, 24, 1024)]):
        step = TrainingStep(ctx, 4 * seq, hidden, 32000, seq=seq)
        got = measure(step, layers, seq)
        jobs["h"][j], jobs["l"][j], jobs["s"][j] = hidden, layers, seq
        jobs["P"][j] = float(layers * (1 + step.experts) * hidden * hidden + hidden * step.vocab)
        jobs["tau"][j], jobs["k_bwd"][j] = np.float32(got["tau"]), np.float32(got["k_bwd"])
        jobs["w"][j] = np.float32(3.0 * got["tau"])
        print(f"hidden {hidden}, {layers} layers, {seq} tokens a sample: tau {got['tau'] * 1e3:.2f} ms, k_bwd {got['k_bwd']:.2f}")
        del step
    dense = measure(DenseStep(ctx, 4 * 1024, 1280, 32000), 24, 1024)
    print(f"without experts, from labels: hidden 1280, 24 layers, 1024 tokens a sample: tau {dense['tau'] * 1e3:.2f} ms, k_bwd {dense['k_bwd']:.2f}")
    n_nodes = 4
    d_out = torch.empty(3 * rb.ASSIGN_DTYPE.itemsize, dtype=torch.uint8, device="cuda:0")
    steps, _ = ctx.schedule_round(rb.to_device(rb.pack_jobs(jobs)), 3, n_nodes, 1 << 20, d_out)
    ctx.sync()
    for j, a in enumerate(rb.from_device(d_out, rb.ASSIGN_DTYPE)):
        print(f"job {j}: {a['g']} GPUs, {a['c']} cores, plan {a['plan']}, {a['thr']:.1f} samples/s")
    ctx.close()


if __name__ == "__main__":
    main()
