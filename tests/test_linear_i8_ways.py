"""The 8-bit linear layer on each way that its calls can take: the kernels are
chosen from sizes alone (checks.cpp), so these sizes are chosen by the way they
take.  References and tolerances are those of test_linear_i8.py.
"""
from __future__ import annotations

import os
import shutil

import numpy as np
import pytest

import paper_2608_23048_amd as roi
from tests.gpu_helpers import f32
from tests.test_linear_i8 import assert_grad, grad_inputs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23048_amd", "csrc")
gpu = pytest.mark.gpu


def test_loads_past_a_sum_stay_in_reach(tmp_path):
    """The offsets of the 256-tile gradient's int8 loads, over whole sums and the
    steps fetched past their ends, on the host."""
    pytest.importorskip("tests.test_sanitizers")
    from tests.test_sanitizers import HERE, SAN, build_and_run
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    exe = tmp_path / "linear_reach_driver"
    out = build_and_run([gxx, "-std=c++17", *SAN, "-Wall", "-Wextra", "-Werror", f"-I{CSRC}",
                         os.path.join(HERE, "linear_reach_driver.cpp"), "-o", str(exe)], exe,
                        tmp_path)
    assert "linear reach ok" in out


# (tokens, rows, cols, weight or input gradient): 256-tiles whose sums are one
# step, end within a step, and are cut into parts
SUM_ENDS = [(64, 4000, 3584, True), (40, 4000, 3588, True), (2100, 1032, 4096, True),
            (1032, 2100, 4096, False)]


@gpu
@pytest.mark.parametrize("tokens,rows,cols,by_tokens", SUM_ENDS)
def test_grads_at_the_end_of_a_sum(tokens, rows, cols, by_tokens):
    """Three steps past its end are fetched, and count for nothing: neighbours of
    the operands in memory are NaN and the largest integers."""
    import torch
    dy, q, s = grad_inputs(tokens, rows, cols, tokens, by_tokens)

    def among(a, fill):
        buf = torch.full((a.numel() + 512 * cols,), fill, dtype=a.dtype, device="cuda")
        buf[:a.numel()] = a.reshape(-1).cuda()
        return buf[:a.numel()].view(a.shape)

    fn = roi.linear_i8_grad_weight if by_tokens else roi.linear_i8_grad_input
    got = fn(among(dy, float("nan")), among(torch.from_numpy(q), 127),
             among(torch.from_numpy(s), float("nan")))
    d = dy.float().numpy()
    assert_grad(f32(got.float()), d if by_tokens else np.ascontiguousarray(d.T), q, s,
                f"{tokens}x{rows}x{cols}")
