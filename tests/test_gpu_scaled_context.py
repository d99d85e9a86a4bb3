"""The calls on e4m3 rows next to a context: both take the same codes and scales, the calls run on the context's plan."""
import pytest
import torch

import paper_2607_18002_b200 as moe

from gpu_util import REL_L2_8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k,H,I", [(5, 16, 4, 256, 128), (300, 8, 2, 512, 256), (64, 64, 8, 768, 384)])
def test_a_context_and_the_calls_run_the_same_layer(T, E, k, H, I):
    g = torch.Generator("cuda").manual_seed(T)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    w1 = moe.scaled_quantize_weights(normal(E, 2 * I, H).mul_(H ** -0.5).bfloat16())
    w2 = moe.scaled_quantize_weights(normal(E, H, I).mul_(I ** -0.5).bfloat16())
    x, x_scale = moe.scaled_quantize(normal(T, H).bfloat16())
    ids, w = moe.choose_experts(normal(T, E), k, scores="sigmoid", bias=0.05 * normal(E), scale=1.5)
    ctx = moe.Context(E, k, H, I, T, max_ops=1, dtype=moe.MOE_DTYPE_FP8_E4M3)
    op = ctx.bind(moe.MOE_CLASS_DECODE, x.view(torch.uint8), ids, w, w1[0].view(torch.uint8), w2[0].view(torch.uint8), x_scale=x_scale, s_gate_up=w1[1], s_down=w2[1])
    ctx.plan(0, op)
    ctx.run([0], fuse_combine=True)
    ctx.check()
    xs = moe.sort_rows(x, op.sorted_to_flat, op.flat_to_sorted, k)
    scales = moe.sort_rows(x_scale, op.sorted_to_flat, op.flat_to_sorted, k)
    a = moe.scaled_swiglu(xs, scales, *w1, op.offsets)
    y = moe.merge_rows(moe.scaled_product(*a, *w2, op.offsets), op.flat_to_sorted, w)
    # the context divides by 448 where the calls multiply, and its activation is rounded elsewhere: a code here and there
    assert torch.linalg.norm(op.y.float() - y.float()) <= REL_L2_8 * torch.linalg.norm(y.float())
