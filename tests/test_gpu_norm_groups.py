"""Block norm's gate gradient where a group's rows lie in several of the blocks' runs of rows: groups shorter than two runs
(kept whole), of a few (joined by a warp) and of very many (joined by a block), with a ragged last group."""
import pytest

from gpu_util import has_cuda
import test_gpu_train_ops as ops

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_cuda(), reason="needs a CUDA device")]
ctx = ops.ctx

CASES = [(2191, cols, dtype, dtype, "group", dict(group=group, tanh=group % 2 == 0))
         for cols, dtype in ((768, "fp32"), (200, "bf16"), (2304, "fp16"), (771, "bf16"))
         for group in (2, 4, 5, 9, 16, 33, 100, 2190)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-%d" % (c[1], c[2], c[5]["group"]))
def test_block_norm_groups_of_every_length(ctx, case):
    ops.test_block_norm_forward_and_backward(ctx, case)
