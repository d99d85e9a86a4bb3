"""What a product of e4m3 rows leaves when a wait inside its kernel runs out: rows that are right, or that say that they are not."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2607_18002_b200 as moe
from paper_2607_18002_b200 import build as moe_build

SOURCE = os.path.join(os.path.dirname(moe.__file__), "csrc", "moe_scaled_product.cu")


def _code():
    with open(SOURCE) as f:
        return re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", f.read()))


def test_nothing_is_given_back_that_was_waited_for_in_vain():
    """A warp that gave up does not arrive on the barriers that let partials and scales be overwritten: the other warps may not have read them yet.  Every hand-over behind a
    wait in the same step asks for its answer."""
    code = _code()
    epilogue = code[code.index("const auto next_partial"):code.index("if (warp == kTmaWarp)")]
    waits = list(re.finditer(r"(next_partial|next_scales)\(\)", epilogue))
    gives = list(re.finditer(r"(if \(ok\) )?(hand_back|scales_read)\(\);", epilogue))
    assert len(gives) == 8
    for g in gives:
        wait = "next_partial" if g[2] == "hand_back" else "next_scales"
        before = max(w.end() for w in waits if w[1] == wait and w.end() < g.start())
        between = epilogue[before:g.start()]
        # ... directly, or by a loop that begins with it, or by the loads in between that are left out
        assert g[1] or "if (!ok) break;" in between or re.search(r"&& ok; (\+\+b|b0 \+= 2)\)", between), epilogue[before - 40:g.end()]


@pytest.fixture(scope="module")
def impatient(tmp_path_factory):
    """The products built from sources in which the roles' waits ask without being suspended and have a limit that the test sets: a healthy launch then gives up here and there.
    (The waits for copies and products in flight keep their limit.)"""
    at = tmp_path_factory.mktemp("impatient")
    header, limits = os.path.relpath(os.path.join(os.path.dirname(moe.__file__), "..", "include"), at), 0
    for name in os.listdir(moe_build.CSRC):
        with open(os.path.join(moe_build.CSRC, name)) as f:
            text = f.read().replace("mbarrier.try_wait", "mbarrier.test_wait").replace('"../../include/', f'"{header}/')
        if name in ("moe_grouped.cuh", "moe_scaled_product.cu"):
            text, n = re.subn(r"gtime_ns\(\) - start > kWaitNs", "gtime_ns() - start > role_wait_ns", text)
            text, m = re.subn(r"i < 64; \+\+i\)\n( +)if \((kTry|__all_sync)", r"i < 2; ++i)\n\1if (\2", text)
            assert n == m == 1, name
            limits += 1
        (at / name).write_text(text)
    assert limits == 2
    source, lib = at / "impatient.cu", at / "impatient.so"
    source.write_text('__device__ volatile unsigned long long role_wait_ns = 2000000000ull;\n#include "moe_scaled_product.cu"\n'
                      'extern "C" int set_role_wait(unsigned long long ns) { return (int)cudaMemcpyToSymbol(role_wait_ns, &ns, sizeof(ns)); }\n')
    built = subprocess.run([moe_build.NVCC, *moe_build.FLAGS, "-o", str(lib), str(source)], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-2000:]
    L, own = ctypes.CDLL(str(lib)), moe.lib()
    for name in ("moe_scaled_product", "moe_scaled_swiglu"):
        getattr(L, name).argtypes = getattr(own, name).argtypes
    L.set_role_wait.argtypes = [ctypes.c_uint64]
    return L


def _at(t):
    return t.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [20, 100])                   # an expert: the forms of one CTA alone, for few rows and of 128 rows
@pytest.mark.parametrize("K", [128, 1024])
def test_rows_are_right_or_say_that_they_are_not(impatient, rows, K):
    E, I, N = 64, 512, 1024
    R = E * rows
    g = torch.Generator("cuda").manual_seed(rows + K)
    codes, scales = moe.scaled_quantize(torch.randn(R, K, device="cuda", generator=g))
    w, ws = moe.scaled_quantize_weights(torch.randn(E, 2 * I, K, device="cuda", generator=g))
    assert N == 2 * I
    offsets = torch.arange(0, R + 1, rows, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    out = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    act, act_scales = torch.empty(R, I, dtype=torch.uint8, device="cuda"), torch.empty(R, I // 128, device="cuda")
    operands = (_at(codes), _at(scales), _at(w), _at(ws), _at(offsets), R, E)

    def launch(limit):
        assert impatient.set_role_wait(limit) == 0
        out.fill_(1.0); act.fill_(0); act_scales.fill_(1.0)
        assert impatient.moe_scaled_product(*operands, N, K, moe.MOE_DTYPE_BF16, _at(out), stream) == moe.MOE_OK
        assert impatient.moe_scaled_swiglu(*operands, I, K, _at(act), _at(act_scales), stream) == moe.MOE_OK
        torch.cuda.synchronize()
        return out.clone(), act.view(R, I // 128, 128).clone(), act_scales.clone()

    want = launch(2_000_000_000)
    assert not torch.isnan(want[0]).any() and not torch.isnan(want[2]).any()
    assert torch.equal(want[0], moe.scaled_product(codes, scales, w, ws, offsets))
    gone, kept = [0, 0], [0, 0]
    for limit in [0, 100, 200, 400, 800, 1200, 1600, 2000, 2500, 3000, 4000, 6000, 10000] * 4:
        y, a, s = launch(limit)
        lost, dead = torch.isnan(y), torch.isnan(s)
        assert torch.equal(torch.where(lost, want[0], y), want[0])
        assert torch.equal(torch.where(dead, want[2], s), want[2])
        assert torch.equal(torch.where(dead[..., None], want[1], a), want[1])
        for i, m in enumerate((lost, dead)):
            gone[i] += int(m.sum())
            kept[i] += int((~m).sum())
    print("gave up, done:", gone, kept)
    assert min(gone) > 0 and min(kept) > 0                    # both have been seen
