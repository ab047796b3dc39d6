"""The product of 8-bit floats on each way that its calls can take: the kernels are
chosen from sizes alone (checks.cpp), so these sizes are chosen by the way they take.
References are those of test_f8.py: small integers and moderate scales, so that all
sums are exact in any order and y is their nearest bf16.
"""
from __future__ import annotations

import os
import shutil

import pytest
import torch

import paper_2608_23048_amd as roi
from tests.test_f8 import E4, E5, E8, blocks, strided

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23048_amd", "csrc")

# (tokens, rows, cols, way): "few" is linear_f8_few_kernel, of which at most 8, at most
# 16 and more tokens, fewer rows than 8192 and more (above 16 tokens: up to 256 blocks of
# 16 rows and 32 tokens, and more) are kernels of their own; else the tile's size
# ("alone": one tile a compute unit), whether tiles are whole or their sums cut, and
# whether a block goes through more than one ("rounds").
WAYS = [
    (3, 8200, 200, "few"), (8, 8193, 1025, "few"), (5, 300, 1664, "few"), (13, 8201, 129, "few"),
    (16, 9000, 640, "few"), (11, 333, 1100, "few"), (31, 257, 640, "few"), (32, 9000, 257, "few"),
    (17, 4128, 127, "few"), (45, 500, 900, "few"), (70, 2101, 131, "few"),
    (1500, 1600, 256, "128 alone whole"), (1038, 32, 65, "128 alone whole"),
    (520, 5000, 1100, "128 alone whole"), (1101, 33, 1938, "128 alone cut"),
    (1030, 1030, 9000, "128 alone cut"), (385, 8487, 67, "128 whole"), (2060, 2060, 6001, "128 whole"),
    (525, 13086, 67, "128 whole rounds"), (4200, 4200, 300, "128 whole rounds"),
    (41, 11079, 16590, "128 cut"), (7237, 1135, 1679, "128 whole cut rounds"),
    (776, 14425, 663, "256 whole"), (5027, 5658, 518, "256 whole rounds"),
    (5000, 5000, 2000, "256 whole rounds"), (130, 8585, 11980, "256 cut"),
    (1193, 13147, 1711, "256 whole cut rounds"),
]


def test_checks_and_ways_under_sanitizers(tmp_path):
    pytest.importorskip("tests.test_sanitizers")
    from tests.test_sanitizers import HERE, SAN, build_and_run
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("g++ or the HIP headers not available")
    want = [f"{t} {r} {c}: {way}" for t, r, c, way in WAYS]
    (tmp_path / "ways.txt").write_text("".join(w.split(":")[0] + "\n" for w in want))
    exe = tmp_path / "f8_checks_driver"
    out = build_and_run([gxx, "-std=c++17", *SAN, "-Wall", "-Wextra", "-Werror",
                         "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                         f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                         os.path.join(CSRC, "checks.cpp"),
                         os.path.join(HERE, "f8_checks_driver.cpp"), "-o", str(exe)], exe,
                        tmp_path)
    assert out.splitlines() == want + ["f8 checks ok"]


def integers(rows, cols, dtype, g):
    return torch.randint(-2, 3, (rows, cols), generator=g, device="cuda").float().to(dtype)


def scales(rows, cols, g):
    s = torch.full((rows, roi.block_scales(cols)), 127, dtype=torch.uint8, device="cuda")
    s[:, : blocks(cols)] = torch.randint(124, 131, (rows, blocks(cols)), generator=g, device="cuda")
    return s.view(E8)


def values(q, s, square):
    """What q and its scales stand for, in 64 bits."""
    e = s.view(torch.uint8)[:, : blocks(q.shape[1])].long()
    power = ((e + 1023 - 127) << 52).view(torch.float64).repeat_interleave(128, 1)[:, : q.shape[1]]
    if square:
        power = power.repeat_interleave(128, 0)[: q.shape[0]]
    return q.double() * power


def nearest(x):
    assert torch.equal(x.float().double().nan_to_num(0), x.nan_to_num(0))
    return x.float().bfloat16()


def same(got, want):
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))


def operands(tokens, rows, cols, dtype, square, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (integers(tokens, cols, dtype, g), scales(tokens, cols, g), integers(rows, cols, E4, g),
            scales(blocks(rows) if square else rows, cols, g))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,rows,cols,way", WAYS)
def test_product_each_way(tokens, rows, cols, way):
    """Both formats, scales of rows and of squares, with and without a bias, NaN between
    the rows and in one row of either operand."""
    for dtype, square in ((E4, True), (E5, False)):
        xq, xs, wq, ws = operands(tokens, rows, cols, dtype, square, tokens + rows)
        b = (torch.arange(rows, device="cuda") % 7 - 3).bfloat16() if dtype == E5 else None
        if dtype == E5:
            xq.view(torch.uint8)[tokens - 1, cols - 1] = 0x7F
            wq.view(torch.uint8)[rows // 2, 0] = 0x7F
        want = torch.mm(values(xq, xs, False), values(wq, ws, square).t().contiguous())
        if b is not None:
            want += b.double()
        y = roi.linear_f8(strided(xq, 1), xs, strided(wq), ws, bias=b)
        assert same(y, nearest(want))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,rows,cols,way", [w for w in WAYS if "cut" in w[3]])
def test_parts_stay_in_the_workspace(tokens, rows, cols, way):
    """A workspace of just the size asked for, full of NaN; one byte less is refused."""
    xq, xs, wq, ws = operands(tokens, rows, cols, E4, True, cols)
    need = roi.linear_f8_workspace(tokens, rows, cols)
    assert need > 0
    work = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    want = roi.linear_f8(strided(xq), xs, strided(wq), ws)
    flat = torch.full((tokens * rows + 300,), 9.0, dtype=torch.bfloat16, device="cuda")
    out = flat[:tokens * rows].view(tokens, rows)
    roi.linear_f8(strided(xq), xs, strided(wq), ws, out=out, workspace=work[:need])
    assert torch.equal(out, want)
    assert bool((work[need:] == 0xFF).all()) and bool((flat[tokens * rows:] == 9).all())
    with pytest.raises(roi.RoiError, match="workspace"):
        roi.linear_f8(strided(xq), xs, strided(wq), ws, workspace=work[:need - 16])


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,rows,cols", [(1101, 33, 1938), (130, 8585, 11980), (1193, 13147, 1711)])
def test_two_graphs_in_turn(tokens, rows, cols):
    """Two captured calls that share a workspace, replayed one after the other between
    eager calls with it, are the eager products."""
    data = [operands(tokens, rows, cols, E4, True, n) for n in range(2)]
    data = [(strided(x), xs, strided(w), ws) for x, xs, w, ws in data]
    want = [roi.linear_f8(*d) for d in data]
    work = torch.empty(roi.linear_f8_workspace(tokens, rows, cols), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graphs, outs = [], []
    for d in data:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(roi.linear_f8(*d, workspace=work))
        graphs.append(graph)
    for turn in range(3):
        for o in outs:
            o.zero_()
        for graph in graphs:
            graph.replay()
        assert torch.equal(roi.linear_f8(*data[turn % 2], workspace=work), want[turn % 2])
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@pytest.mark.gpu
def test_tiles_of_a_batch_cut_at_any_token():
    """A token's result is the same in another batch, the way taken being another's."""
    tokens, rows, cols = 1500, 1600, 256
    xq, xs, wq, ws = operands(tokens, rows, cols, E4, True, 5)
    xq, wq = strided(xq), strided(wq)
    whole = roi.linear_f8(xq, xs, wq, ws)
    for first in (1, 33, 400, 1029):
        assert torch.equal(roi.linear_f8(xq[first:], xs[first:], wq, ws), whole[first:])
        assert torch.equal(roi.linear_f8(xq[:first], xs[:first], wq, ws), whole[:first])


@pytest.mark.gpu
def test_a_plan_keeps_its_memory():
    """A parameter and its gradient that get new memory after the plan was made: the plan
    steps the memory that they had, which nobody else gets meanwhile."""
    p, g = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    old = p.detach()
    avg, sq = roi.adamw_moments(p)
    plan = roi.adamw_plan([(p, g, avg, sq)])
    address = g.data_ptr()
    p.data = torch.full((1000,), 5.0, device="cuda")
    del g
    other = [torch.full((1000,), float("nan"), device="cuda") for _ in range(8)]
    assert address not in [t.data_ptr() for t in other]
    roi.adamw_grouped(plan, roi.adamw_params(0.5, t=1))
    # 1 (1 - 0.5 0.05) - 0.5 g / (|g| + eps), the default decay being 0.05; its fp32
    # operations are within 2^-20
    assert bool(((old - 0.475).abs() < 2.0 ** -20).all()) and bool((p == 5).all())


@pytest.mark.gpu
def test_streams_of_every_way_at_once():
    """Calls on two streams, each with a workspace of its own."""
    shapes = [(16, 9000, 640), (1101, 33, 1938), (4200, 4200, 300), (130, 8585, 11980)]
    calls = []
    for t, r, c in shapes:
        xq, xs, wq, ws = operands(t, r, c, E5, False, t)
        calls.append((strided(xq), xs, strided(wq), ws))
    want = [roi.linear_f8(*a) for a in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for turn in range(3):
        for n, a in enumerate(calls):
            with torch.cuda.stream(streams[(n + turn) % 2]):
                outs.append((n, roi.linear_f8(*a)))
    torch.cuda.synchronize()
    for n, y in outs:
        assert torch.equal(y, want[n])


def far_apart(q, stride):
    """q in rows `stride` bytes apart, NaN between them."""
    room = torch.full((q.shape[0], stride), 0x7F, dtype=torch.uint8, device="cuda")
    room[:, : q.shape[1]] = q.view(torch.uint8)
    return room.view(q.dtype)[:, : q.shape[1]]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,rows,cols,x_stride,w_stride,way", [
    (70000, 33000, 200, 65536, 131072, "256"),     # y past 2^31 values, both operands past 2^32 bytes
    (5, 1100000, 100, 1 << 22, 4096, "few"),       # the weight past 2^32 bytes
    (1500, 1600, 256, 1 << 22, 1 << 22, "128"),    # the widest strides
    (776, 14425, 663, 1 << 22, 1 << 20, "256"),
])
def test_products_past_32_bits(tokens, rows, cols, x_stride, w_stride, way):
    xq, xs, wq, ws = operands(tokens, rows, cols, E4, False, 8)
    y = roi.linear_f8(far_apart(xq, x_stride), xs, far_apart(wq, w_stride), ws)
    at = [t for t in (0, 1, 255, 256, 32767, 32768, 65074, 65075, 65076, 65535, 65536, tokens - 2, tokens - 1)
          if t < tokens]
    x, w = values(xq, xs, False)[at], values(wq, ws, False).t().contiguous()
    assert same(y[at], nearest(torch.mm(x, w)))


@pytest.mark.gpu
def test_product_without_a_sum():
    """No columns: the bias, or zeros; more blocks than a launch takes are refused."""
    b = torch.arange(70, device="cuda").bfloat16()
    for tokens in (1, 40, 3000):
        xq, wq = (torch.empty(n, 0, dtype=E4, device="cuda") for n in (tokens, 70))
        none = torch.empty(tokens, 0, dtype=E8, device="cuda"), torch.empty(70, 0, dtype=E8, device="cuda")
        assert torch.equal(roi.linear_f8(xq, none[0], wq, none[1], bias=b), b.expand(tokens, 70))
        assert not bool(roi.linear_f8(xq, none[0], wq, none[1]).any())


def test_too_many_blocks_without_a_sum():
    most = (1 << 30) - 1
    assert roi.lib().roi_linear_f8_workspace(most, 1, 0) == roi.ROI_E_UNSUPPORTED
    assert roi.lib().roi_linear_f8_workspace(1 << 28, 1, 0) == 0
    with pytest.raises(roi.RoiError, match="elements"):
        roi.linear_f8_workspace(most, 70, 0)
