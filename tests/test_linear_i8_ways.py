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
from tests.gpu_helpers import bf16_bits, f32
from tests.test_linear_i8 import (assert_grad, dev, expand, grad_inputs, meta_of, random_2of4,
                                  to_bf16)

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


# (tokens, rows, cols, 2:4, way): "few" is linear_few_kernel, of which at most 8,
# at most 16 and more tokens, fewer rows than 8192 and more, and rows that end
# within 16 bytes are kernels of their own, and above 16 tokens up to 256 blocks of
# 16 rows and 32 tokens, and more; else the tile's size ("alone": one tile a
# compute unit), whether tiles are whole or their sums cut, and whether rows are
# copied first.
LINEAR_WAYS = [
    (1, 8192, 96, False, "few"), (8, 8201, 272, False, "few"), (5, 9001, 77, False, "few"),
    (9, 8192, 128, False, "few"), (16, 8999, 400, False, "few"), (13, 8209, 131, False, "few"),
    (1, 8192, 96, True, "few"), (7, 8201, 288, True, "few"), (16, 8999, 416, True, "few"),
    (8, 333, 1040, False, "few"), (16, 331, 1041, False, "few"), (12, 331, 1056, True, "few"),
    (17, 4112, 99, False, "few"), (31, 5001, 1031, False, "few"), (32, 4201, 144, False, "few"),
    (20, 4113, 160, True, "few"), (70, 2101, 131, False, "few"), (101, 1903, 176, False, "few"),
    (101, 1903, 192, True, "few"), (40, 333, 259, False, "few"), (33, 333, 288, True, "few"),
    (1101, 301, 1008, False, "128 alone whole"), (1101, 301, 1024, True, "128 alone whole"),
    (1101, 301, 1001, False, "128 alone whole copied"),
    (1101, 131, 8192, False, "128 alone cut"), (1101, 131, 8192, True, "128 alone cut"),
    (1025, 129, 8111, False, "128 alone cut copied"),
    (4095, 4399, 160, False, "128 whole"), (4095, 4399, 160, True, "128 whole"),
    (4095, 4399, 157, False, "128 whole copied"),
    (1665, 4837, 4192, False, "128 whole cut"), (1365, 991, 8832, True, "128 cut"),
    (2199, 4111, 288, False, "256 whole"), (2199, 4111, 288, True, "256 whole"),
    (2199, 4111, 283, False, "256 whole copied"),
    (2499, 1701, 9000, False, "256 cut copied"), (2499, 1701, 8992, True, "256 cut"),
    (4241, 3957, 2048, True, "256 whole cut"), (4094, 4351, 4096, False, "256 whole cut"),
]
# (operation, tokens, rows, cols, way): "ready" converts the int8 operand first,
# "deep" has a tile a compute unit.
GRAD_WAYS = [
    ("weight", 64, 4000, 3584, "256 whole"), ("weight", 40, 4000, 3588, "ready whole"),
    ("weight", 2100, 1032, 4096, "256 cut"), ("input", 1032, 2100, 4096, "256 cut copied"),
    ("input", 461, 7807, 4662, "256 cut copied"), ("weight", 1746, 983, 4432, "256 cut copied"),
    ("weight", 130, 2100, 2500, "128 whole copied"), ("input", 2500, 130, 2100, "128 whole copied"),
    ("weight", 710, 4613, 3515, "ready whole cut copied"),
    ("input", 3358, 556, 4776, "ready whole cut copied"),
    ("weight", 1000, 257, 260, "deep cut copied"), ("input", 257, 1000, 260, "deep cut copied"),
    ("weight", 2000, 256, 1024, "deep cut"), ("input", 256, 2000, 1024, "deep cut"),
    ("weight", 333, 96, 256, "deep whole"), ("input", 333, 96, 256, "deep whole"),
]


def test_sizes_take_these_ways(tmp_path):
    pytest.importorskip("tests.test_sanitizers")
    from tests.test_sanitizers import HERE, SAN, build_and_run
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("g++ or the HIP headers not available")
    want = [f"linear {t} {r} {c} {int(p)}: {way}" for t, r, c, p, way in LINEAR_WAYS]
    want += [f"{op} {t} {r} {c} 0: {way}" for op, t, r, c, way in GRAD_WAYS]
    (tmp_path / "ways.txt").write_text("".join(w.split(":")[0] + "\n" for w in want))
    exe = tmp_path / "linear_ways_driver"
    out = build_and_run([gxx, "-std=c++17", *SAN, "-Wall", "-Wextra", "-Werror",
                         "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                         f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                         os.path.join(CSRC, "checks.cpp"),
                         os.path.join(HERE, "linear_ways_driver.cpp"), "-o", str(exe)], exe,
                        tmp_path)
    assert out.splitlines() == want + ["linear ways ok"]


@gpu
@pytest.mark.parametrize("tokens,rows,cols,packed,way", LINEAR_WAYS)
def test_linear_each_way(tokens, rows, cols, packed, way):
    """The documented sequence bit for bit, with and without a bias, both types.
    The sums are below 2^53 and so exact in 64 bits."""
    import torch
    rng = np.random.default_rng(tokens * 31 + rows)
    xq = dev(rng.integers(-128, 128, (tokens, cols)).astype(np.int8))
    xs = dev(rng.uniform(1e-3, 1, tokens).astype(np.float32))
    ws = dev(rng.uniform(1e-4, 1e-2, rows).astype(np.float32))
    b, meta = to_bf16(rng.standard_normal(rows)).cuda(), None
    if packed:
        values, idx = random_2of4(rng, rows, cols)
        wq, dense, meta = dev(values), dev(expand(values, idx, cols)), dev(meta_of(idx).view(np.int32))
    else:
        dense = wq = dev(rng.integers(-128, 128, (rows, cols)).astype(np.int8))
    total = torch.mm(xq.double(), dense.double().t().contiguous())
    scaled = total.float() * ws * xs[:, None]
    for bias, want in ((b, scaled + b.float()), (None, scaled)):
        y = roi.linear_i8(xq, xs, wq, ws, meta=meta, bias=bias, dtype=torch.float32)
        assert torch.equal(y, want)
        assert np.array_equal(bf16_bits(roi.linear_i8(xq, xs, wq, ws, meta=meta, bias=bias)),
                              bf16_bits(want.bfloat16()))


@gpu
@pytest.mark.parametrize("op,tokens,rows,cols,way", GRAD_WAYS)
def test_grads_each_way(op, tokens, rows, cols, way):
    by_tokens = op == "weight"
    dy, q, s = grad_inputs(tokens, rows, cols, tokens + cols, by_tokens)
    fn = roi.linear_i8_grad_weight if by_tokens else roi.linear_i8_grad_input
    got = fn(dy.cuda(), dev(q), dev(s))
    d = dy.float().numpy()
    assert_grad(f32(got.float()), d if by_tokens else np.ascontiguousarray(d.T), q, s,
                f"{op} {tokens}x{rows}x{cols}")


@gpu
@pytest.mark.parametrize("tokens", [1101, 2300])
def test_exported_layer_at_many_tokens(tokens):
    """mask_export at 2:4, quantized: the compressed product equals the dense one
    bit for bit through the tiles."""
    import torch
    from paper_2608_23048_amd import workloads as wl
    rows, cols = 300, 416
    W, logits, _ = wl.small_case(rows, cols, 3, device="cuda")
    Wm, vals, _, meta = roi.mask_export(logits, W, 2, 4, want_meta=True)
    dq, ds = roi.quantize_rows(Wm)
    pq, ps = roi.quantize_rows(vals.view(rows, cols // 2))
    xq, xs = roi.quantize_rows(torch.randn(tokens, cols, device="cuda").bfloat16())
    b = torch.randn(rows, device="cuda").bfloat16()
    assert torch.equal(roi.linear_i8(xq, xs, dq, ds, bias=b),
                       roi.linear_i8(xq, xs, pq, ps, meta=meta, bias=b))


# ------------------------------------------------------------------ workspaces
MOST_TOKENS, MOST = (1 << 30) - 1, (1 << 22) - 1


@pytest.mark.parametrize("tokens,rows,cols,packed,status", [
    (40, 8, 131072, 0, roi.ROI_E_UNSUPPORTED),   # a sum that may pass 32 bits
    (1100, 8, 131104, 1, roi.ROI_E_UNSUPPORTED),
    (0, 0, 131072, 0, roi.ROI_E_UNSUPPORTED),
    (40, 8, 48, 1, roi.ROI_E_INVAL),             # 2:4 rows end within a metadata word
    (MOST_TOKENS, MOST, 64, 0, roi.ROI_E_UNSUPPORTED),  # more blocks than a launch
    (-1, 8, 64, 0, roi.ROI_E_INVAL), (1 << 30, 8, 64, 0, roi.ROI_E_UNSUPPORTED),
])
def test_workspace_refuses_what_the_product_refuses(tokens, rows, cols, packed, status):
    L = roi.lib()
    assert L.roi_linear_i8_workspace(tokens, rows, cols, packed) == status
    assert L.roi_last_error()
    with pytest.raises(roi.RoiError) as e:
        roi.linear_i8_workspace(tokens, rows, cols, bool(packed))
    assert e.value.status == status


@pytest.mark.parametrize("name", ["linear_i8_grad_weight", "linear_i8_grad_input"])
def test_workspace_refuses_what_the_gradients_refuse(name):
    L = roi.lib()
    fn = getattr(L, f"roi_{name}_workspace")
    sizes = (64, MOST, MOST) if name.endswith("weight") else (MOST_TOKENS, 64, MOST)
    assert fn(*sizes) == roi.ROI_E_UNSUPPORTED and L.roi_last_error()
    assert fn(64, 1 << 22, 64) == roi.ROI_E_UNSUPPORTED
    assert fn(64, -1, 64) == roi.ROI_E_INVAL
    with pytest.raises(roi.RoiError, match="too many elements"):
        getattr(roi, name + "_workspace")(*sizes)
    assert fn(64, 64, 64) >= 0 and not L.roi_last_error()


@gpu
def test_refused_product_allocates_nothing():
    import torch
    q = torch.zeros(3000, 131073, dtype=torch.int8, device="cuda")
    s = torch.ones(3000, device="cuda")
    out = torch.empty(3000, 3000, dtype=torch.bfloat16, device="cuda")
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    with pytest.raises(roi.RoiError, match="exact int32 sum") as e:
        roi.linear_i8(q, s, q, s, out=out)
    assert e.value.status == roi.ROI_E_UNSUPPORTED
    assert torch.cuda.max_memory_allocated() == held


# ------------------------------------------------------------------ alignments
def test_alignments_that_calls_take(tmp_path):
    pytest.importorskip("tests.test_sanitizers")
    from tests.test_sanitizers import HERE, SAN, build_and_run
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("g++ or the HIP headers not available")
    exe = tmp_path / "linear_align_driver"
    out = build_and_run([gxx, "-std=c++17", *SAN, "-Wall", "-Wextra", "-Werror",
                         "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                         f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                         os.path.join(CSRC, "checks.cpp"),
                         os.path.join(HERE, "linear_align_driver.cpp"), "-o", str(exe)], exe,
                        tmp_path)
    assert "linear alignments ok" in out


@gpu
@pytest.mark.parametrize("cut", [333, 1102, 5])
def test_batch_cut_at_any_token(cut):
    """Rows from any token on, through the product at few and many tokens, and both
    gradients: as of copies of them, whose scales start at 16 bytes."""
    import torch
    tokens, rows, cols = 2300, 264, 144
    xq, xs = roi.quantize_rows(torch.randn(tokens, cols, device="cuda"))
    wq, ws = roi.quantize_rows(torch.randn(rows + cut, cols, device="cuda"))
    gy = torch.randn(tokens, rows, device="cuda").bfloat16()
    assert xs[cut:].data_ptr() % 16 and ws[cut:].data_ptr() % 16
    parts = (xq[cut:], xs[cut:], wq[cut:], ws[cut:])
    whole = [p.clone() for p in parts]
    for count in (tokens - cut, 70, 9):
        few = [parts[0][:count], parts[1][:count], *parts[2:]]
        assert torch.equal(roi.linear_i8(*few),
                           roi.linear_i8(whole[0][:count], whole[1][:count], *whole[2:]))
    assert torch.equal(roi.linear_i8_grad_weight(gy[cut:], *parts[:2]),
                       roi.linear_i8_grad_weight(gy[cut:], *whole[:2]))
    assert torch.equal(roi.linear_i8_grad_input(gy, *parts[2:]),
                       roi.linear_i8_grad_input(gy, *whole[2:]))


# ------------------------------------------------------- the type's largest rows
@gpu
@pytest.mark.parametrize("cols", [1, 9, 1025, 8193, 20000, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_at_the_largest_values(cols, dtype):
    """Rows that hold the type's lowest or largest value (a mask's, say) and their
    neighbours come back finite, half a step off at most (q is within 2^-14 of a
    step of x / scale, and the restored value is rounded once more)."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    top = torch.finfo(t).max
    x = torch.randn(6, cols).to(t)
    x[0, -1], x[1, 0], x[2, cols // 2] = torch.finfo(t).min, top, 2.0 ** 127
    x[3] = top
    x[4, 0] = top * (1 - torch.finfo(t).eps)
    x[5] = torch.finfo(t).min
    q, s = roi.quantize_rows(x.cuda())
    back = roi.dequantize_rows(q, s, dtype=t)
    assert torch.isfinite(s).all() and torch.isfinite(back).all()
    want, got, step = x.double(), back.cpu().double(), s.cpu().double()[:, None]
    off = (got - want).abs()
    assert (off <= step * (0.5 + 2.0 ** -14) + got.abs() * torch.finfo(t).eps / 2).all()
    assert (q[3] == 127).all() and (q[5] == -127).all()
