"""Linear layers, dropout, block norms and the head's cross entropy together: a step of a dense model against automatic
differentiation of the same model in double precision, its masks, and the step in a captured graph."""
import numpy as np
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
from paper_2408_08586_b200 import workloads
import product_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]


@pytest.fixture(scope="module")
def ctx():
    return rb.Context(workloads.ENV, device=0)


def model(p, x, label, keep, tied):
    """-> cross entropies, in double precision"""
    import torch
    norm = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5) * w  # noqa: E731
    x = x * keep[0]
    a = ref.act(norm(x, p["w_in"]) @ p["w_up"] + p["b_up"], "gelu")
    x = x + (a @ p["w_down"] + p["b_down"]) * keep[1]
    z = norm(x, p["w_out"]) @ (p["w_head"].t() if tied else p["w_head"])
    live = label >= 0
    nll = torch.logsumexp(z, 1) - z.gather(1, label.long().clamp(min=0)[:, None])[:, 0]
    return torch.where(live, nll, 0.0)


@pytest.mark.parametrize("tied,drop", [(True, 0.1), (False, 0.4), (True, 0.0)])
def test_gradients_of_a_dense_step_are_those_of_its_model(ctx, tied, drop):
    """Half precision.  Some ten tensors on the way of a gradient are rounded to 2^-11 of their entries, the slope of gelu is taken
    at a rounded place (off by at most 1.2 |pre| 2^-11), and the norms' backward passes at most double what comes in:
    ten times two times 2^-10 is below 2^-5, of a gradient's norm."""
    import torch
    from paper_2408_08586_b200.training_step import DENSE_PARAMETERS, DenseStep, draw_labels
    step = DenseStep(ctx, 150, 72, 1000, inner=200, drop=drop, tied=tied, dtype=torch.float16, seed=5)
    step.advance()
    x, label = draw_labels(step, 3)
    label[7] = -1
    w = torch.rand(150, device="cuda") + 0.5
    nll = step.forward(x, label).clone()
    got = {k: v.clone() for k, v in step.backward(w).items()}
    keep = [ref.keep(s, 150, 72, drop) for s in step.seed.tolist()]
    assert step.seed.tolist() == [[5, 2], [5, 3]] and (drop == 0 or not torch.equal(keep[0], keep[1]))
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in step.p.items()}
    x64 = x.double().cpu().requires_grad_()
    want_nll = model(p, x64, label.cpu(), keep, tied)
    leaves = [p[k] for k in DENSE_PARAMETERS] + [x64]
    want = dict(zip(DENSE_PARAMETERS + ("x",), torch.autograd.grad((w.double().cpu() * want_nll).sum(), leaves)))
    assert float((nll.double().cpu() - want_nll.detach()).norm()) <= 2.0 ** -7 * float(want_nll.detach().norm()) and nll[7] == 0
    assert set(got) == set(want)
    for name, g in got.items():
        off = float((g.double().cpu() - want[name]).norm())
        assert off <= 2.0 ** -5 * float(want[name].norm()), name
    # the head in one call gives the same step
    again_nll, again = step.step(x, label, w)
    assert float((again_nll - nll).abs().max()) <= 2.0 ** -18 * float(nll.abs().max())
    for name, g in again.items():
        assert float((g.double() - got[name].double()).norm()) <= 2.0 ** -9 * float(got[name].double().norm()), name


def test_a_captured_dense_step_draws_new_masks(ctx):
    import torch
    from paper_2408_08586_b200.training_step import DenseStep, draw_labels
    stream = torch.cuda.Stream()
    own = rb.Context(workloads.ENV, device=0, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        step = DenseStep(own, 200, 128, 3000, drop=0.3)
        x, label = draw_labels(step)
        step.advance()
        step.step(x, label)
        stream.synchronize()
        step.seed.copy_(torch.tensor([[0, 0], [0, 1]]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step.advance()
            step.step(x, label)
        seen = []
        for _ in range(3):
            graph.replay()
            stream.synchronize()
            seen.append({k: v.clone() for k, v in step.g.items()} | {"nll": step.b["nll"].clone(), "x": step.b["dx"].clone(), "mask": step.b["x"] == 0})
        assert step.seed.tolist() == [[0, 6], [0, 7]]
        assert not torch.equal(seen[0]["mask"], seen[1]["mask"]) and not torch.equal(seen[1]["nll"], seen[2]["nll"])
        # replayed under the first masks: the same bits; and called outside of the graph
        step.seed.copy_(torch.tensor([[0, 0], [0, 1]]))
        graph.replay()
        stream.synchronize()
        first = {k: v.clone() for k, v in step.g.items()} | {"nll": step.b["nll"].clone(), "x": step.b["dx"].clone()}
        step.step(x, label)
        stream.synchronize()
        for k, v in first.items():
            assert torch.equal(v, seen[0][k]), k
            assert torch.equal(v, step.g[k] if k in step.g else step.b["nll"] if k == "nll" else step.b["dx"]), k
    own.sync()
    del graph
    own.close()


def test_scratch_of_products_does_not_grow_in_a_capture(ctx):
    import torch
    stream = torch.cuda.Stream()
    own = rb.Context(workloads.ENV, device=0, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        h, w = torch.zeros(300, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(5000, 64, dtype=torch.bfloat16, device="cuda")
        label, loss = torch.zeros(300, dtype=torch.int32, device="cuda"), torch.zeros(300, device="cuda")
        y = torch.zeros(8, device="cuda")
        desc = rb.head_loss(300, 64, 5000, torch.bfloat16, by_output=True)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(rb.RubickError) as e:
                own.head_loss_step(desc, h, w, label, None, loss, None, torch.empty_like(h), torch.empty_like(w))
            assert e.value.code == rb.ESTATE
            y += 1
        graph.replay()
        own.head_loss_step(desc, h, w, label, None, loss, None, torch.empty_like(h), torch.empty_like(w))
        stream.synchronize()
        assert (y == 1).all() and abs(float(loss[0]) - np.log(5000)) < 1e-5
    own.sync()
    del graph
    own.close()


def test_a_dense_profile_is_measured(ctx):
    from paper_2408_08586_b200 import training_step as ts
    before = rb.kernel_launches()
    got = ts.measure(ts.DenseStep(ctx, 256, 256, 1000), layers=12, seq=64, repeats=2)
    assert rb.kernel_launches() - before >= 5 * 10
    assert 0 < got["tau"] < 10 and 0 < got["k_bwd"] < 100
