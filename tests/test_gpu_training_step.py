"""The training-step operators together: gradients of a whole step against automatic differentiation of the same model in
double precision, the combined head against the separate one, and the measured profile through the scheduler."""
import numpy as np
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
from paper_2408_08586_b200 import workloads

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]


@pytest.fixture(scope="module")
def ctx():
    return rb.Context(workloads.ENV, device=0)


def model(step, p, x, index, teacher, token_weight):
    """The step's loss in double precision; the experts chosen and the counts are the step's."""
    import torch

    def norm(v, w):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5) * w

    def edge(x, y, w_after, gate, w_before):
        g = torch.tanh(gate).repeat_interleave(step.edge.group_rows, 0)[: len(x)]
        x = x + step.edge.alpha * g * norm(y, w_after)
        return x, norm(x, w_before)

    h0 = norm(x, p["w_in"])
    x1, h1 = edge(x, h0 @ p["w_block"], p["w_after1"], p["gate1"], p["w_before2"])
    probs = torch.softmax(h1 @ p["w_router"], 1)
    chosen = step.b["index"].long()
    weight = torch.gather(probs, 1, chosen)
    weight = weight / weight.sum(1, keepdim=True)
    y2 = torch.zeros_like(h1)
    for j in range(step.chosen):
        y2 = y2 + weight[:, j:j + 1] * torch.einsum("nd,nde->ne", h1, p["w_expert"][chosen[:, j]])
    x2, h2 = edge(x1, y2, p["w_after2"], p["gate2"], p["w_before3"])
    T = step.loss.temperature
    q = torch.softmax(teacher.double() / T, 1)
    log_p = torch.gather(torch.log_softmax(h2 @ p["w_head"] / T, 1), 1, index.long())
    kd = T * T * (q * (q.log() - log_p)).sum(1)
    n = step.route.group_rows
    balance = torch.stack([step.experts * ((step.b["counts"][g].double() / (step.chosen * len(part))) * part.mean(0)).sum()
                           for g, part in enumerate(probs.split(n))]).mean()
    return kd, step.coef * balance, (token_weight.double() * kd).sum() + step.coef * balance


def test_gradients_of_a_step_are_those_of_its_model(ctx):
    """Single precision throughout.  The step's products round at 2^-24 of sums of up to 96 terms, some dozen operations deep,
    and the norms divide by numbers near one: 2^-14 of a gradient's largest entry is allowed."""
    import torch
    from paper_2408_08586_b200.training_step import TrainingStep, draw_batch
    torch.backends.cuda.matmul.allow_tf32 = False
    step = TrainingStep(ctx, 60, 96, 257, seq=25, experts=6, chosen=2, teacher=9, dtype=torch.float32)
    x, index, teacher = draw_batch(step, 3)
    w = torch.rand(60, device="cuda") + 0.5
    kd, balance = (t.clone() for t in step.forward(x, index, teacher))
    got = {k: v.clone() for k, v in step.backward(w).items()}
    p = {k: v.detach().double().requires_grad_() for k, v in step.p.items()}
    x64 = x.double().requires_grad_()
    want_kd, want_balance, value = model(step, p, x64, index, teacher, w)
    want = dict(zip(list(p) + ["x"], torch.autograd.grad(value, list(p.values()) + [x64])))
    assert float((kd - want_kd.detach()).abs().max()) <= 2.0 ** -14 * float(want_kd.detach().abs().max())
    assert abs(float(balance) - float(want_balance.detach())) <= 2.0 ** -14 * float(want_balance.detach())
    for name, g in got.items():
        off = float((g.double() - want[name]).abs().max())
        assert off <= 2.0 ** -14 * float(want[name].abs().max()), name
    # the head's loss and gradient in one kernel give the same step
    kd2, balance2, again = step.step(x, index, teacher, w)
    assert float((kd2 - kd).abs().max()) <= 2.0 ** -18 * float(kd.abs().max()) and torch.equal(balance2, balance)
    for name, g in again.items():
        assert float((g - got[name]).abs().max()) <= 2.0 ** -14 * float(got[name].abs().max()), name


def test_a_measured_profile_goes_through_the_scheduler(ctx):
    import torch
    from paper_2408_08586_b200 import training_step as ts
    cfg = workloads.make("paper-scale", J=2)
    c = rb.Context(cfg["env"], device=0)
    plans, _ = rb.enumerate_plans(cfg["g_levels"])
    c.set_space(plans, cfg["g_levels"], cfg["c_levels"], cfg["m_levels"])
    step = ts.TrainingStep(c, 256, 256, 1000, seq=64)
    before = rb.kernel_launches()
    got = ts.measure(step, layers=12, seq=64, repeats=2)
    assert rb.kernel_launches() - before >= 5 * 10          # the library's kernels ran, forward and backward
    assert 0 < got["tau"] < 10 and 0 < got["k_bwd"] < 100
    for j in range(2):
        cfg["jobs"]["tau"][j], cfg["jobs"]["k_bwd"][j] = np.float32(got["tau"]), np.float32(got["k_bwd"])
    d_out = torch.zeros(2 * rb.ASSIGN_DTYPE.itemsize, dtype=torch.uint8, device="cuda:0")
    c.schedule_round(rb.to_device(rb.pack_jobs(cfg["jobs"])), 2, 1, 1 << 20, d_out)
    c.sync()
    out = rb.from_device(d_out, rb.ASSIGN_DTYPE)
    assert (out["status"] == rb.RUNNING).any() and (out["thr"][out["status"] == rb.RUNNING] > 0).all()
    c.close()
