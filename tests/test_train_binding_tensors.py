"""What a descriptor's first call looks for in its tensors, seen from the host alone."""
import pytest
import torch

from paper_2408_08586_b200 import binding as rb


def _context():
    """A context that has no library behind it: whatever gets past the look over its tensors is refused by the entry point."""
    c = object.__new__(rb.Context)
    c._h, c.device = None, -1                              # (-1: where torch says that CPU tensors are)
    return c


def _tensors(rows=4, cols=8, k=2):
    f, i, b = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.float32, torch.int32, torch.bfloat16))
    return dict(x=b(rows, cols), w=b(cols), f2=f(rows, 2), fc=f(cols), index=i(rows, k), weight=f(rows, k), counts=i(1, cols), sums=f(1, cols), valid=i(1),
                one=f(1), n=f(rows), mask=torch.ones(rows, dtype=torch.uint8), teacher=f(rows, k))


CALLS = {
    "block_norm_forward": ("norm", ["x", "x", "w", "x", "w", "x", "x", "f2"]),
    "block_norm_backward": ("norm", ["x", "x", "w", "x", "w", "f2", "x", "x", "x", "x", "fc", "x", "fc"]),
    "router_forward": ("router", ["x", "mask", "index", "weight", "counts", "sums", "valid", "one"]),
    "router_backward": ("router", ["x", "index", "weight", "counts", "valid", "one", "weight", "x"]),
    "distill_forward": ("distill", ["x", "index", "teacher", "n", "n"]),
    "distill_backward": ("distill", ["x", "index", "teacher", "n", "n", "x"]),
    "distill_step": ("distill", ["x", "index", "teacher", "n", "n", "n", "x"]),
}
DESCS = {"norm": lambda: rb.block_norm(4, 8, torch.bfloat16), "router": lambda: rb.router(4, 8, 2, torch.bfloat16),
         "distill": lambda: rb.distill(4, 8, 2, torch.bfloat16, torch.float32)}


@pytest.mark.parametrize("method", CALLS)
def test_tensors_of_another_type_layout_or_device_are_refused(method):
    op, names = CALLS[method]
    good = _tensors()
    call = lambda c, d, args: getattr(c, method)(d, *args)  # noqa: E731
    c, desc = _context(), DESCS[op]()
    for _ in range(2):                                     # as it should be: it gets as far as the entry point
        with pytest.raises(rb.RubickError) as e:
            call(c, desc, [good[n] for n in names])
        assert e.value.code == rb.EINVAL and "null context" in str(e.value)
    for at, name in enumerate(names):
        t = good[name]
        bad = [(t.to(torch.float64), "type"), (t.to(torch.float16), "type")]
        if t.dim() == 2 and min(t.shape) > 1:
            bad.append((t.t().contiguous().t(), "strides"))
        for wrong, word in bad:
            with pytest.raises(rb.RubickError) as e:
                call(c, DESCS[op](), [wrong if i == at else good[n] for i, n in enumerate(names)])
            assert e.value.code == rb.EINVAL and word in str(e.value), (name, word)
        c.device = 0                                        # these tensors are not there
        with pytest.raises(rb.RubickError) as e:
            call(c, DESCS[op](), [good[n] if i == at else None for i, n in enumerate(names)])
        assert "cuda:0" in str(e.value)
        c.device = -1
