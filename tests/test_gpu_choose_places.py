"""Routers by scores on operands at every place that their documentation allows (addresses of elements)."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe
from tests import scaled_util as su

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_choose.cu")


def test_what_is_read_by_four_is_known_to_be_aligned_to_four():
    """Everything that the kernels load or store by four elements has its address looked at where the form is chosen."""
    with open(SOURCE) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    kernels, forms = code[code.index("choose_kernel("):], re.findall(r"const bool vec = ([^;]*);", code)
    by_four = {"choose_kernel": {"row": "logits", "a.bias": "bias"}, "choose_grad_kernel": {"z_row": "logits", "out": "d_logits"}}
    used = set(re.findall(r"load_row<\w+, kPer, kVec>\(([\w.]+),", kernels)) | set(re.findall(r"store4\((\w+) \+", kernels))
    assert used == {v for k in by_four.values() for v in k}
    for form, names in zip(forms, by_four.values(), strict=True):
        assert set(re.findall(r"misaligned\((\w+),", form)) == set(names.values()), form


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,k,groups,top_groups", [(4, 2, 1, 1), (64, 6, 8, 3), (256, 8, 1, 1), (256, 8, 8, 4), (512, 8, 4, 2), (1024, 20, 1, 1)])
def test_a_bias_that_is_a_slice(kind, E, k, groups, top_groups):
    g = torch.Generator().manual_seed(E)
    buf = (torch.randn(E + 8, generator=g) * 0.1).cuda()
    for dtype in (torch.float32, torch.bfloat16):
        z = (torch.randn(70, E, generator=g) * 1.5).to(dtype).cuda()
        z64 = su.to_numpy(z)
        for at in (1, 2, 3, 4):
            bias = buf[at:at + E]
            ids, w = moe.choose_experts(z, k, scores=kind, bias=bias, groups=groups, top_groups=top_groups)
            want = su.chosen(z64, k, kind, bias.cpu().numpy(), groups, top_groups)
            assert np.array_equal(ids.cpu().numpy(), want)
            ref = su.weights_of(z64, want, kind, True, 1.0)
            assert np.all(np.abs(su.to_numpy(w) - ref) <= su.weights_error(z64, want, kind) * np.abs(ref) + 2.0 ** -120)
            same = moe.choose_experts(z, k, scores=kind, bias=bias.clone(), groups=groups, top_groups=top_groups)
            assert torch.equal(ids, same[0])
