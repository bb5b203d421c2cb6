"""The training-step operators in captured CUDA graphs: what a graph holds stays valid when later calls need more scratch."""
import pytest

from gpu_util import has_cuda
from paper_2408_08586_b200 import binding as rb
from paper_2408_08586_b200 import workloads
import test_gpu_train_ops as ops

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]


def calls(ctx, rows, cols, experts):
    """(run, outputs) of a block norm's backward pass and a router's forward pass, both of which use scratch"""
    import torch
    s, opt, desc = ops.norm_case(rows, cols, "bf16", "bf16", "group", group=rows // 3 + 1)
    rstd = torch.full((rows, 2), 0.7, device="cuda")
    grads = [torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(cols, device="cuda"), torch.empty_like(s["gate"]), torch.empty(cols, device="cuda")]
    z, mask, ropt, rdesc = ops.router_case(rows, experts, 4, "fp32", group=rows // 2 + 1)
    o = ops.router_outputs(rows, experts, 4, 2)

    def run():
        ctx.block_norm_backward(desc, s["x"], s["y"], s["w_after"], s["gate"], s["w_before"], rstd, s["dx_out"], s["dh"], *grads)
        ctx.router_forward(rdesc, z, mask, o["index"], o["weight"], o["counts"], o["prob_sum"], o["valid"], o["loss"])
    return run, grads + list(o.values())


def test_a_captured_graph_outlives_larger_calls():
    import torch
    stream = torch.cuda.Stream()
    ctx = rb.Context(workloads.ENV, device=0, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        run, outs = calls(ctx, 2000, 520, 40)
        large, large_outs = calls(ctx, 9000, 8192, 800)
        run()
        stream.synchronize()
        want = [v.clone() for v in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for _ in range(2):
            for v in outs:
                v.zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(v, w) for v, w in zip(outs, want))
            large()                                        # grows the scratch that the graph uses
        held = [torch.full((1 << 24,), 3.0, device="cuda") for _ in range(8)]
        stream.synchronize()
        assert all((v == 3).all() for v in held)
    ctx.sync()
    del graph
    ctx.close()


def test_scratch_does_not_grow_in_a_capture():
    """A call that would have to allocate is refused; the capture itself goes on."""
    import torch
    stream = torch.cuda.Stream()
    ctx = rb.Context(workloads.ENV, device=0, stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        run, outs = calls(ctx, 2000, 520, 40)
        x, y = torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y.add_(x)
            with pytest.raises(rb.RubickError) as e:
                run()
            assert e.value.code == rb.ESTATE and "capture" in str(e.value)
            y.add_(x)
        graph.replay()
        run()
        stream.synchronize()
        assert (y == 2).all() and torch.isfinite(outs[2]).all()
    ctx.sync()
    del graph
    ctx.close()
