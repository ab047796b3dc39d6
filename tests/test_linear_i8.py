"""The 8-bit linear layer around a masked weight: quantize_rows,
dequantize_rows, linear_i8 (dense and 2:4 weights) and its two gradients.

The quantizer and the product are fixed sequences of IEEE fp32 operations over
exact integers, so they are compared bit for bit with numpy.  The gradients sum
in fp32 in an order of the kernel's own: with A = sum_k |dy| |x^| (x^ the bf16
operand, formed as documented), a sum of K products and its partial sums are off
by at most K 2^-23 A (one rounding of at most 2^-23, truncation included, for
each addition), and the result's rounding to bf16 by 2^-8 of its value.
"""
from __future__ import annotations

import numpy as np
import pytest

import paper_2608_23048_amd as roi
from tests.gpu_helpers import bf16_bits, bf16_rne_bits, f32

FAKE = 0x7F0000000000  # 16-byte aligned, never dereferenced: every call below fails validation
GB = 1 << 30


# ------------------------------------------------------------ refusals (CPU)
@pytest.fixture(scope="module")
def L():
    return roi.lib()


def quantize_call(L, fn="roi_quantize_rows", **kw):
    a = dict(x=FAKE, dtype=0, rows=4, cols=8, q=FAKE + GB, scale=FAKE + 2 * GB)
    a.update(kw)
    if fn == "roi_quantize_rows":
        return L.roi_quantize_rows(a["x"], a["dtype"], a["rows"], a["cols"], a["q"], a["scale"],
                                   None)
    return L.roi_dequantize_rows(a["q"], a["scale"], a["rows"], a["cols"], a["x"], a["dtype"], None)


@pytest.mark.parametrize("fn", ["roi_quantize_rows", "roi_dequantize_rows"])
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), roi.ROI_E_INVAL), (dict(dtype=-1), roi.ROI_E_INVAL),
    (dict(rows=-1), roi.ROI_E_INVAL), (dict(cols=-1), roi.ROI_E_INVAL),
    (dict(rows=1 << 31), roi.ROI_E_UNSUPPORTED), (dict(cols=1 << 31), roi.ROI_E_UNSUPPORTED),
    (dict(x=None), roi.ROI_E_INVAL), (dict(q=None), roi.ROI_E_INVAL),
    (dict(scale=None), roi.ROI_E_INVAL), (dict(x=FAKE + 8), roi.ROI_E_INVAL),
    (dict(q=FAKE + GB + 4), roi.ROI_E_INVAL), (dict(scale=FAKE + 2 * GB + 4), roi.ROI_E_INVAL),
    (dict(q=FAKE + 48), roi.ROI_E_INVAL),            # q inside x
    (dict(scale=FAKE + 16), roi.ROI_E_INVAL),        # scale inside x
    (dict(scale=FAKE + GB + 16), roi.ROI_E_INVAL),   # scale inside q
])
def test_rows_reject_before_launch(L, fn, kw, status):
    if fn == "roi_dequantize_rows" and kw == dict(scale=FAKE + GB + 16):
        pytest.skip("two inputs may overlap")
    assert quantize_call(L, fn, **kw) == status
    assert L.roi_last_error()


def test_rows_with_nothing_to_do(L):
    assert quantize_call(L, rows=0, x=None, q=None, scale=None) == roi.ROI_OK
    for kw in (dict(rows=0, x=None, q=None, scale=None), dict(cols=0, x=None, q=None)):
        assert quantize_call(L, "roi_dequantize_rows", **kw) == roi.ROI_OK


def linear_call(L, **kw):
    a = dict(xq=FAKE, xs=FAKE + GB, wq=FAKE + 2 * GB, meta=None, ws=FAKE + 3 * GB, bias=None,
             tokens=4, rows=8, cols=64, y=FAKE + 4 * GB, dtype=0, work=None, bytes=0)
    a.update(kw)
    return L.roi_linear_i8(a["xq"], a["xs"], a["wq"], a["meta"], a["ws"], a["bias"], a["tokens"],
                           a["rows"], a["cols"], a["y"], a["dtype"], a["work"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), roi.ROI_E_INVAL), (dict(tokens=-1), roi.ROI_E_INVAL),
    (dict(rows=-1), roi.ROI_E_INVAL), (dict(cols=-64), roi.ROI_E_INVAL),
    (dict(tokens=1 << 31), roi.ROI_E_UNSUPPORTED), (dict(rows=1 << 22), roi.ROI_E_UNSUPPORTED),
    (dict(cols=131072), roi.ROI_E_UNSUPPORTED),      # 2^17 products of (-128)^2 are 2^31
    (dict(xq=None), roi.ROI_E_INVAL), (dict(xs=None), roi.ROI_E_INVAL),
    (dict(wq=None), roi.ROI_E_INVAL), (dict(ws=None), roi.ROI_E_INVAL),
    (dict(y=None), roi.ROI_E_INVAL), (dict(xq=FAKE + 8), roi.ROI_E_INVAL),
    (dict(bias=FAKE + 5 * GB + 2), roi.ROI_E_INVAL), (dict(y=FAKE + 32), roi.ROI_E_INVAL),
    (dict(y=FAKE + 3 * GB + 16), roi.ROI_E_INVAL),
    (dict(meta=FAKE + 5 * GB, cols=48), roi.ROI_E_INVAL),
    (dict(meta=FAKE + 5 * GB + 4), roi.ROI_E_INVAL),
    (dict(meta=FAKE + 4 * GB + 16), roi.ROI_E_INVAL),  # under y
    (dict(bytes=-1), roi.ROI_E_INVAL),
])
def test_linear_rejects_before_launch(L, kw, status):
    assert linear_call(L, **kw) == status
    assert L.roi_last_error()


def test_linear_with_nothing_to_do(L):
    assert linear_call(L, tokens=0, xq=None, xs=None, y=None) == roi.ROI_OK
    assert linear_call(L, rows=0, wq=None, ws=None, y=None) == roi.ROI_OK
    assert L.roi_linear_i8_workspace(-1, 4, 4, 0) < 0
    assert L.roi_linear_i8_workspace(4, 4, 4, 0) >= 0


def grad_call(L, fn, **kw):
    a = dict(dy=FAKE, q=FAKE + GB, s=FAKE + 2 * GB, tokens=4, rows=8, cols=16, out=FAKE + 3 * GB,
             work=None, bytes=0)
    a.update(kw)
    return getattr(L, fn)(a["dy"], a["q"], a["s"], a["tokens"], a["rows"], a["cols"], a["out"],
                          a["work"], a["bytes"], None)


GRADS = ["roi_linear_i8_grad_weight", "roi_linear_i8_grad_input"]


@pytest.mark.parametrize("fn", GRADS)
@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), roi.ROI_E_INVAL), (dict(rows=-2), roi.ROI_E_INVAL),
    (dict(cols=-1), roi.ROI_E_INVAL), (dict(rows=1 << 22), roi.ROI_E_UNSUPPORTED),
    (dict(cols=1 << 22), roi.ROI_E_UNSUPPORTED), (dict(tokens=1 << 31), roi.ROI_E_UNSUPPORTED),
    (dict(dy=None), roi.ROI_E_INVAL), (dict(q=None), roi.ROI_E_INVAL),
    (dict(s=None), roi.ROI_E_INVAL), (dict(out=None), roi.ROI_E_INVAL),
    (dict(dy=FAKE + 2), roi.ROI_E_INVAL), (dict(out=FAKE + 16), roi.ROI_E_INVAL),
    (dict(out=FAKE + GB), roi.ROI_E_INVAL), (dict(out=FAKE + 2 * GB), roi.ROI_E_INVAL),
    (dict(bytes=-5), roi.ROI_E_INVAL),
])
def test_grads_reject_before_launch(L, fn, kw, status):
    assert grad_call(L, fn, **kw) == status
    assert L.roi_last_error()


@pytest.mark.parametrize("fn", GRADS)
def test_grads_with_nothing_to_do(L, fn):
    assert grad_call(L, fn, cols=0, q=None, out=None) == roi.ROI_OK
    assert getattr(L, fn + "_workspace")(-1, 1, 1) < 0


def test_host_tensors_are_refused():
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: roi.quantize_rows(x), lambda: roi.dequantize_rows(q, s),
                 lambda: roi.linear_i8(q, s, q, s), lambda: roi.linear_i8_grad_weight(x, q, s),
                 lambda: roi.linear_i8_grad_input(x, q, s)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError):
        roi.quantize_rows(x.half())
    with pytest.raises(TypeError):
        roi.quantize_rows([1.0])


def test_checks_and_plans_under_sanitizers(tmp_path):
    import os
    import shutil
    pytest.importorskip("tests.test_sanitizers")
    from tests.test_sanitizers import CSRC, HERE, ROOT, SAN, build_and_run
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("g++ or the HIP headers not available")
    exe = tmp_path / "linear_checks_driver"
    out = build_and_run([gxx, "-std=c++17", *SAN, "-Wall", "-Wextra", "-Werror",
                         "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                         f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                         os.path.join(CSRC, "checks.cpp"),
                         os.path.join(HERE, "linear_checks_driver.cpp"), "-o", str(exe)], exe,
                        tmp_path)
    assert "linear checks ok" in out


# ------------------------------------------------------------------ references
FLOOR = np.float32(2.0 ** -126)


def quantize_ref(x):
    """(q, scale) by the documented fp32 sequence."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(axis=1, initial=0).astype(np.float32)
        bad = ~np.isfinite(x).all(axis=1)
        amax = np.where(bad, np.float32(1), amax)
        s = (amax / np.float32(127)).astype(np.float32)
        low = ~(s > FLOOR)
        inv = np.where(low, np.float32(2.0 ** 126),
                       np.float32(127) * (np.float32(1) / np.where(low, np.float32(1), amax)))
        q = np.rint(np.where(bad[:, None], 0, x) * inv[:, None].astype(np.float32))
    s = np.where(bad, np.float32(np.nan), np.where(low, FLOOR, s)).astype(np.float32)
    return np.where(bad[:, None], 0, q).astype(np.int8), s


def bf16_of(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32)


def linear_ref(xq, xs, wq, ws, bias=None):
    """fp32 result by the documented sequence (bias: bf16 patterns)."""
    total = xq.astype(np.int64) @ wq.astype(np.int64).T
    with np.errstate(all="ignore"):
        y = total.astype(np.float32) * ws[None, :].astype(np.float32)
        y = y * xs[:, None].astype(np.float32)
        return y if bias is None else y + bf16_of(bias)[None, :]


def grad_refs(dy, q, s):
    """(sum_k dy[k, d] x^[k, c] in fp64, sum of magnitudes, K) with x^ the bf16
    rounding of the fp32 product s q."""
    xh = bf16_of(bf16_rne_bits((q.astype(np.float32) * s[:, None]).astype(np.float32)))
    dy, xh = dy.astype(np.float64), xh.astype(np.float64)
    return dy.T @ xh, np.abs(dy).T @ np.abs(xh), dy.shape[0]


def assert_grad(got, dy, q, s, what):
    """dy [K, D], q [K, C], s [K]; got [D, C] (fp32 values of the bf16 result)."""
    ref, mag, K = grad_refs(dy, q, s)
    slack = K * 2.0 ** -23 * mag
    bound = slack + 2.0 ** -8 * (np.abs(ref) + slack) + 2.0 ** -133
    err = np.abs(got.astype(np.float64) - ref)
    assert got.shape == ref.shape and np.all(err <= bound), (
        f"{what}: {int((err > bound).sum())} of {ref.size} off, worst "
        f"{float((err - bound).max()):.3g}")


def expand(values, idx, cols):
    """Dense int8 rows from 2:4 values [rows, cols / 2] and indices [groups, 2]."""
    rows = values.shape[0]
    dense = np.zeros((rows * cols // 4, 4), np.int8)
    np.put_along_axis(dense, idx.astype(np.int64), values.reshape(-1, 2), axis=1)
    return dense.reshape(rows, cols)


def meta_of(idx):
    nib = (idx[:, 0].astype(np.uint32) | (idx[:, 1].astype(np.uint32) << 2)).reshape(-1, 8)
    return (nib << (4 * np.arange(8, dtype=np.uint32))).sum(axis=1, dtype=np.uint32)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def to_bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def random_2of4(rng, rows, cols):
    values = rng.integers(-128, 128, (rows, cols // 2)).astype(np.int8)
    pairs = np.array([(i, j) for i in range(4) for j in range(i + 1, 4)], np.uint8)
    return values, pairs[rng.integers(0, 6, rows * cols // 4)]


# ------------------------------------------------------------------- GPU tests
gpu = pytest.mark.gpu
COLS = [1, 7, 8, 63, 512, 2047, 2048, 2049, 4865, 8192, 8193, 32768, 32769]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_rows_bit_exact(cols, dtype):
    import torch
    rng = np.random.default_rng(cols)
    rows = 9
    x = rng.standard_normal((rows, cols)).astype(np.float32) * np.float32(3)
    x[1] = 0
    x[2, cols // 2] = 300           # one value far above the others
    x[3] *= np.float32(1e-36)       # scales around the floor
    x[4] *= np.float32(1e-41)
    x[5] *= np.float32(1e37)
    x[6] = np.where(np.arange(cols) % 2, 2.0, 1.0)  # x = amax / 2: ties at 63.5
    x[7, cols - 1] = np.inf
    x[8, 0] = np.nan
    t = to_bf16(x) if dtype == "bf16" else torch.from_numpy(x)
    q, s = roi.quantize_rows(t.cuda())
    back = {d: roi.dequantize_rows(q, s, dtype=d) for d in (torch.bfloat16, torch.float32)}
    q0, s0 = quantize_ref(t.float().numpy())
    assert np.array_equal(q.cpu().numpy(), q0)
    assert np.array_equal(s.cpu().numpy().view(np.uint32) & 0x7FFFFFFF,
                          s0.view(np.uint32) & 0x7FFFFFFF)
    prod = q0.astype(np.float32) * s0[:, None]
    ok = np.isfinite(s0)
    assert np.array_equal(f32(back[torch.float32])[ok].view(np.uint32), prod[ok].view(np.uint32))
    assert np.array_equal(bf16_bits(back[torch.bfloat16])[ok], bf16_rne_bits(prod[ok]))
    for b in back.values():
        assert np.isnan(f32(b.float())[~ok]).all()
    # at most half a step off (and the two roundings of x inv and of q s)
    err = np.abs(prod[ok].astype(np.float64) - t.float().numpy()[ok])
    assert np.all(err <= s0[ok, None].astype(np.float64) * (0.5 + 127 * 2.0 ** -21) + 2.0 ** -149)


@gpu
def test_rows_given_outputs_and_empty():
    import torch
    x = torch.randn(5, 33, device="cuda").bfloat16()
    q, s = roi.quantize_rows(x)
    q2, s2 = torch.full_like(q, 99), torch.full_like(s, 99)
    assert roi.quantize_rows(x, out=(q2, s2))[0] is q2
    assert torch.equal(q, q2) and torch.equal(s, s2)
    one, so = roi.quantize_rows(x[0].clone())  # 1-D: one row
    assert torch.equal(one, q[0]) and torch.equal(so, s[:1])
    for shape in ((0, 8), (3, 0)):
        e, se = roi.quantize_rows(torch.empty(shape, device="cuda"))
        assert e.shape == shape and se.shape == (shape[0],)
        assert (se == 2.0 ** -126).all()
        assert roi.dequantize_rows(e, se).shape == shape
    with pytest.raises(ValueError, match="contiguous"):
        roi.quantize_rows(x.t())
    with pytest.raises(ValueError, match="2-D"):
        roi.quantize_rows(x.view(5, 11, 3))
    with pytest.raises(ValueError, match="2-D"):
        roi.dequantize_rows(q.view(5, 11, 3), s)
    with pytest.raises(ValueError, match="shape"):
        roi.quantize_rows(x, out=(q2[:4], s2))
    with pytest.raises(ValueError, match="shape"):
        roi.dequantize_rows(q, s[:3].clone())
    with pytest.raises(roi.RoiError, match="aligned"):
        roi.quantize_rows(x.view(-1)[1:9])


LINEAR = [(1, 1, 1), (1, 16, 128), (2, 17, 129), (15, 33, 100), (16, 64, 896), (17, 48, 257),
          (32, 20, 64), (33, 130, 272), (64, 31, 1000), (65, 129, 128), (127, 128, 144),
          (128, 300, 640), (130, 127, 77), (257, 260, 384), (300, 513, 16)]


@gpu
@pytest.mark.parametrize("tokens,rows,cols", LINEAR)
def test_linear_dense_bit_exact(tokens, rows, cols):
    import torch
    rng = np.random.default_rng(tokens * 7 + rows)
    xq = rng.integers(-128, 128, (tokens, cols)).astype(np.int8)
    wq = rng.integers(-128, 128, (rows, cols)).astype(np.int8)
    xs = rng.uniform(1e-3, 1, tokens).astype(np.float32)
    ws = rng.uniform(1e-4, 1e-2, rows).astype(np.float32)
    b = to_bf16(rng.standard_normal(rows))
    args = [dev(a) for a in (xq, xs, wq, ws)]
    for bias in (None, b):
        want = linear_ref(xq, xs, wq, ws, None if bias is None else bf16_bits(bias))
        y = roi.linear_i8(*args, bias=None if bias is None else bias.cuda(), dtype=torch.float32)
        assert np.array_equal(f32(y).view(np.uint32), want.view(np.uint32))
        y = roi.linear_i8(*args, bias=None if bias is None else bias.cuda())
        assert np.array_equal(bf16_bits(y), bf16_rne_bits(want))


@gpu
@pytest.mark.parametrize("tokens,rows,cols", [(1030, 40, 257), (1100, 300, 1001), (1025, 5, 3)])
def test_linear_of_copied_rows(tokens, rows, cols):
    """Rows that end within 16 bytes, through the tiles."""
    assert roi.linear_i8_workspace(tokens, rows, cols) >= (tokens + rows) * cols
    test_linear_dense_bit_exact(tokens, rows, cols)


PACKED = [(1, 1, 32), (1, 16, 256), (3, 17, 96), (16, 40, 896), (17, 33, 288), (40, 64, 128),
          (64, 130, 512), (65, 128, 160), (130, 129, 1024), (200, 260, 352), (300, 48, 32)]


@gpu
@pytest.mark.parametrize("tokens,rows,cols", PACKED)
def test_linear_2of4_bit_exact(tokens, rows, cols):
    import torch
    rng = np.random.default_rng(tokens + 11 * rows)
    xq = rng.integers(-128, 128, (tokens, cols)).astype(np.int8)
    values, idx = random_2of4(rng, rows, cols)
    xs = rng.uniform(1e-3, 1, tokens).astype(np.float32)
    ws = rng.uniform(1e-4, 1e-2, rows).astype(np.float32)
    b = to_bf16(rng.standard_normal(rows))
    want = linear_ref(xq, xs, expand(values, idx, cols), ws, bf16_bits(b))
    args = [dev(a) for a in (xq, xs, values, ws)]
    meta = dev(meta_of(idx).view(np.int32))
    y = roi.linear_i8(*args, meta=meta, bias=b.cuda(), dtype=torch.float32)
    assert np.array_equal(f32(y).view(np.uint32), want.view(np.uint32))
    y = roi.linear_i8(*args, meta=meta, bias=b.cuda())
    assert np.array_equal(bf16_bits(y), bf16_rne_bits(want))


@gpu
@pytest.mark.filterwarnings("ignore:overflow:RuntimeWarning")
@pytest.mark.parametrize("cols", [131071, 131056])
@pytest.mark.parametrize("tokens", [1, 12, 30, 70, 300, 1100])
def test_linear_extremes(tokens, cols):
    """The largest sums, rows of zeros with the smallest scale, a NaN row."""
    import torch
    rows = 5
    xq = np.full((tokens, cols), -128, np.int8)
    wq = np.full((rows, cols), -128, np.int8)
    wq[1] = 127
    wq[2] = 0
    xs = np.full(tokens, 2.0 ** -126, np.float32)
    xs[-1] = np.nan
    ws = np.array([1, 2.0 ** 100, 2.0 ** -126, 3e38, 1e-30], np.float32)
    y = f32(roi.linear_i8(dev(xq), dev(xs), dev(wq), dev(ws), dtype=torch.float32))
    want = np.array([128 * 128, -128 * 127, 0, 128 * 128, 128 * 128], np.int64) * cols
    row = (want.astype(np.float32) * ws) * np.float32(2.0 ** -126)
    assert np.array_equal(y[:-1], np.broadcast_to(row, (tokens - 1, rows)))
    assert np.isnan(y[-1]).all()


@gpu
@pytest.mark.parametrize("tokens", [1, 12, 30, 70, 1100])
def test_linear_2of4_longest_sum(tokens):
    """131040 columns, half of them kept, and fields of every value."""
    import torch
    cols, rows = 131040, 6
    rng = np.random.default_rng(tokens)
    xq = np.full((tokens, cols), -128, np.int8)
    xq[-1] = rng.integers(-128, 128, cols)
    values, idx = random_2of4(rng, rows, cols)
    values[:3] = np.array([-128, 127, 1], np.int8)[:, None]
    y = roi.linear_i8(dev(xq), torch.ones(tokens, device="cuda"), dev(values),
                      torch.ones(rows, device="cuda"), meta=dev(meta_of(idx).view(np.int32)),
                      dtype=torch.float32)
    dense = expand(values, idx, cols).astype(np.float64)
    want = xq.astype(np.float64) @ dense.T
    assert np.array_equal(f32(y), want.astype(np.float32))


@gpu
@pytest.mark.parametrize("packed", [False, True])
def test_linear_empty(packed):
    import torch
    z = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda")  # noqa: E731
    o = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    meta = (lambda r, c: torch.zeros(r * c // 32, dtype=torch.int32, device="cuda")
            if packed else None)
    k = 2 if packed else 1
    assert roi.linear_i8(z(0, 32), o(0), z(4, 32 // k), o(4), meta=meta(4, 32)).shape == (0, 4)
    assert roi.linear_i8(z(3, 32), o(3), z(0, 32 // k), o(0), meta=meta(0, 32)).shape == (3, 0)
    b = torch.randn(4, device="cuda").bfloat16()
    for tokens in (3, 100, 1100):  # a sum over nothing is 0: the bias remains
        y = roi.linear_i8(z(tokens, 0), o(tokens), z(4, 0), o(4), meta=meta(4, 0), bias=b)
        assert torch.equal(y, b.expand(tokens, 4))


@gpu
def test_linear_binding_refusals():
    import torch
    xq, wq = (torch.zeros(n, 64, dtype=torch.int8, device="cuda") for n in (3, 5))
    xs, ws = torch.ones(3, device="cuda"), torch.ones(5, device="cuda")
    meta = torch.zeros(10, dtype=torch.int32, device="cuda")
    bad = [
        dict(xq=xq.float()), dict(xq=xq[0]), dict(xq=xq[:, ::2]), dict(xs=xs[:2].clone()),
        dict(ws=xs), dict(xs=xs.double()), dict(wq=wq[:, :32].contiguous()),
        dict(meta=meta), dict(wq=wq[:, :32].contiguous(), meta=meta[:9].clone()),
        dict(bias=torch.zeros(5, device="cuda")), dict(dtype=torch.float16),
        dict(out=torch.zeros(3, 4, device="cuda")), dict(workspace=torch.zeros(4, device="cuda")),
        dict(xs=xs.cpu()), dict(bias=torch.zeros(5, dtype=torch.bfloat16)),
    ]
    for kw in bad:
        with pytest.raises((TypeError, ValueError)):
            roi.linear_i8(**{**dict(xq=xq, xs=xs, wq=wq, ws=ws), **kw})
    q48 = torch.zeros(3, 48, dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError, match="32"):
        roi.linear_i8(q48, xs, q48[:, :24].contiguous(), xs, meta=meta)
    gy = torch.zeros(3, 5, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(grad_y=gy.float()), dict(grad_y=gy[:2].clone()), dict(xs=xs[:1].clone()),
               dict(xq=xq[0]), dict(out=torch.zeros(5, 64, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            roi.linear_i8_grad_weight(**{**dict(grad_y=gy, xq=xq, xs=xs), **kw})
    with pytest.raises(ValueError):
        roi.linear_i8_grad_input(gy, xq, xs)


GRAD = [(1, 1, 1), (3, 17, 5), (64, 128, 128), (65, 136, 132), (63, 120, 124), (130, 129, 131),
        (200, 300, 77), (333, 96, 256), (1000, 257, 260), (128, 8, 520), (70, 520, 4),
        # more 128-tiles than compute units and few sums: two tiles a unit
        (130, 2100, 2500), (2500, 130, 2100)]


def grad_inputs(tokens, rows, cols, seed, by_tokens):
    rng = np.random.default_rng(seed)
    k = tokens if by_tokens else rows
    dy = to_bf16(rng.standard_normal((tokens, rows)) * 1e-3)
    q = rng.integers(-128, 128, (k, cols)).astype(np.int8)
    s = rng.uniform(1e-3, 1, k).astype(np.float32)
    return dy, q, s


@gpu
@pytest.mark.parametrize("by_tokens", [True, False], ids=["weight", "input"])
@pytest.mark.parametrize("tokens,rows,cols", GRAD)
def test_grads(tokens, rows, cols, by_tokens):
    dy, q, s = grad_inputs(tokens, rows, cols, tokens + rows, by_tokens)
    fn = roi.linear_i8_grad_weight if by_tokens else roi.linear_i8_grad_input
    got = fn(dy.cuda(), dev(q), dev(s))
    d = dy.float().numpy()
    assert_grad(f32(got.float()), d if by_tokens else d.T, q, s, f"{tokens}x{rows}x{cols}")
    again = fn(dy.cuda(), dev(q), dev(s))
    assert np.array_equal(bf16_bits(got), bf16_bits(again))


@gpu
@pytest.mark.parametrize("by_tokens", [True, False], ids=["weight", "input"])
@pytest.mark.parametrize("k,d,c", [(1032, 4104, 4092), (1030, 4100, 4093), (2100, 1032, 4096)])
def test_grads_of_many_tiles(k, d, c, by_tokens):
    """More tiles than compute units: the operand converted beforehand, whole
    tiles and cut ones in one call, with and without whole chunks a row."""
    dy, q, s = grad_inputs(*((k, d) if by_tokens else (d, k)), c, k + d, by_tokens)
    fn = roi.linear_i8_grad_weight if by_tokens else roi.linear_i8_grad_input
    need = (roi.linear_i8_grad_weight_workspace(k, d, c) if by_tokens
            else roi.linear_i8_grad_input_workspace(d, k, c))
    assert need >= 2 * k * c
    got = f32(fn(dy.cuda(), dev(q), dev(s)).float())
    dy = dy.float().numpy()
    assert_grad(got, dy if by_tokens else np.ascontiguousarray(dy.T), q, s, f"{k}x{d}x{c}")


@gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("tokens,rows,cols", [(2200, 4112, 288), (500, 4100, 1312),
                                              (4096, 4400, 160), (530, 700, 4000)])
def test_linear_of_many_tiles(tokens, rows, cols, packed):
    import torch
    rng = np.random.default_rng(tokens)
    xq = rng.integers(-128, 128, (tokens, cols)).astype(np.int8)
    xs = rng.uniform(1e-3, 1, tokens).astype(np.float32)
    ws = rng.uniform(1e-4, 1e-2, rows).astype(np.float32)
    meta = None
    if packed:
        wq, idx = random_2of4(rng, rows, cols)
        dense, meta = expand(wq, idx, cols), dev(meta_of(idx).view(np.int32))
    else:
        dense = wq = rng.integers(-128, 128, (rows, cols)).astype(np.int8)
    # products and sums of integers below 2^53 are exact in fp64
    total = xq.astype(np.float64) @ dense.astype(np.float64).T
    want = total.astype(np.float32) * ws[None, :] * xs[:, None]
    args = [dev(a) for a in (xq, xs, wq, ws)]
    y = roi.linear_i8(*args, meta=meta, dtype=torch.float32)
    assert np.array_equal(f32(y).view(np.uint32), want.view(np.uint32))
    assert np.array_equal(bf16_bits(roi.linear_i8(*args, meta=meta)), bf16_rne_bits(want))


@gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("tokens,rows,cols", [(1100, 130, 8192), (4096, 4352, 4096)])
def test_linear_of_cut_sums(tokens, rows, cols, packed):
    """Long sums of few tiles, and a last round of few tiles: cut and added up."""
    import torch
    assert roi.linear_i8_workspace(tokens, rows, cols, packed) > 0
    rng = np.random.default_rng(tokens)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    draw = lambda *n: torch.randint(-128, 128, n, device="cuda", generator=g,  # noqa: E731
                                    dtype=torch.int8)
    xq, xs = draw(tokens, cols), torch.rand(tokens, device="cuda", generator=g)
    ws, meta = torch.rand(rows, device="cuda", generator=g), None
    if packed:
        values, idx = random_2of4(rng, rows, cols)
        wq, dense = dev(values), dev(expand(values, idx, cols))
        meta = dev(meta_of(idx).view(np.int32))
    else:
        dense = wq = draw(rows, cols)
    # products and sums of integers below 2^53 are exact in fp64
    want = torch.mm(xq.double(), dense.double().t().contiguous()).float() * ws * xs[:, None]
    assert torch.equal(roi.linear_i8(xq, xs, wq, ws, meta=meta, dtype=torch.float32), want)
    assert torch.equal(roi.linear_i8(xq, xs, wq, ws, meta=meta), want.bfloat16())


@gpu
def test_grads_against_differences():
    """Both gradients are the slopes of L = sum(grad_y y) along one weight or
    one activation: y is linear in each, so a difference quotient in 64 bits is
    the slope, and the kernels' are within the bf16 roundings of the operand
    (2^-8 of the magnitudes) and of the result."""
    tokens, rows, cols = 37, 24, 40
    dy, xq, xs = grad_inputs(tokens, rows, cols, 5, True)
    _, wq, ws = grad_inputs(tokens, rows, cols, 6, False)
    gw = f32(roi.linear_i8_grad_weight(dy.cuda(), dev(xq), dev(xs)).float())
    gx = f32(roi.linear_i8_grad_input(dy.cuda(), dev(wq), dev(ws)).float())
    d = dy.double().numpy()
    x, w = xq * xs[:, None].astype(np.float64), wq * ws[:, None].astype(np.float64)
    loss = lambda x, w: float((d * (x @ w.T)).sum())  # noqa: E731
    rng = np.random.default_rng(7)
    h = 0.5
    for _ in range(20):
        r, c, t = rng.integers(rows), rng.integers(cols), rng.integers(tokens)
        for got, mag, pert in ((gw[r, c], np.abs(d[:, r]) @ np.abs(x[:, c]), "w"),
                               (gx[t, c], np.abs(d[t]) @ np.abs(w[:, c]), "x")):
            up, dn = (x.copy(), w.copy()), (x.copy(), w.copy())
            i, at = (1, (r, c)) if pert == "w" else (0, (t, c))
            up[i][at] += h
            dn[i][at] -= h
            slope = (loss(*up) - loss(*dn)) / (2 * h)
            tol = (2.0 ** -8 + max(tokens, rows) * 2.0 ** -23) * mag
            assert abs(got - slope) <= tol + 2.0 ** -8 * (abs(slope) + tol) + 1e-9


@gpu
@pytest.mark.parametrize("by_tokens", [True, False], ids=["weight", "input"])
def test_grads_empty_sums_and_nan(by_tokens):
    import torch
    fn = roi.linear_i8_grad_weight if by_tokens else roi.linear_i8_grad_input
    tokens, rows = (0, 6) if by_tokens else (6, 0)
    dy = torch.zeros(tokens, rows, dtype=torch.bfloat16, device="cuda")
    out = torch.full((6, 10), 7.0, dtype=torch.bfloat16, device="cuda")
    fn(dy, torch.zeros(0, 10, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"),
       out=out)
    assert (out == 0).all()
    assert fn(torch.zeros(4, 4, dtype=torch.bfloat16, device="cuda"),
              torch.zeros(4, 0, dtype=torch.int8, device="cuda"),
              torch.ones(4, device="cuda")).shape == (4, 0)
    dy, q, s = grad_inputs(70, 70, 33, 1, by_tokens)
    s[69] = np.nan  # a row that held an infinity: what sums over it is NaN
    got = fn(dy.cuda(), dev(q), dev(s))
    assert torch.isnan(got).all()


@gpu
@pytest.mark.parametrize("tokens,rows,cols", [(70, 45, 77), (300, 257, 144), (1030, 1100, 390)])
def test_padding_and_neighbours_are_left_alone(tokens, rows, cols):
    """Outputs are written exactly; what lies behind them in memory stays, and
    padded (zero) rows give zeros."""
    import torch
    guard = 64

    def framed(n, dtype):
        buf = torch.full((n + guard,), 77, dtype=dtype, device="cuda")
        return buf, buf[:n]

    x = torch.randn(tokens, cols, device="cuda").bfloat16()
    x[50:] = 0
    bq, q = framed(tokens * cols, torch.int8)
    bs, s = framed(tokens, torch.float32)
    q = q.view(tokens, cols)
    roi.quantize_rows(x, out=(q, s))
    wq, ws = roi.quantize_rows(torch.randn(rows, cols, device="cuda"))
    by, y = framed(tokens * rows, torch.bfloat16)
    y = y.view(tokens, rows)
    roi.linear_i8(q, s, wq, ws, out=y)
    bw, gw = framed(rows * cols, torch.bfloat16)
    gy = torch.randn(tokens, rows, device="cuda").bfloat16()
    roi.linear_i8_grad_weight(gy, q, s, out=gw.view(rows, cols))
    bx, gx = framed(tokens * cols, torch.bfloat16)
    roi.linear_i8_grad_input(gy, wq, ws, out=gx.view(tokens, cols))
    bd, xd = framed(tokens * cols, torch.float32)
    roi.dequantize_rows(q, s, out=xd.view(tokens, cols))
    bz, z = framed(tokens * rows, torch.float32)
    roi.linear_i8(q, s, wq, ws, out=z.view(tokens, rows))
    for b in (bq, bs, by, bw, bx, bd, bz):
        assert (b[-guard:] == 77).all()
    assert (y[50:] == 0).all() and (xd.view(tokens, cols)[50:] == 0).all()


# ---------------------------------------------------------- used together
@gpu
def test_exported_layer_dense_and_2of4_agree():
    """mask_export at 2:4, quantized: the compressed product equals the dense
    one bit for bit, at few and at many tokens."""
    import torch
    from paper_2608_23048_amd import workloads as wl
    rows, cols = 160, 416
    W, logits, _ = wl.small_case(rows, cols, 3, device="cuda")
    Wm, vals, idx, meta = roi.mask_export(logits, W, 2, 4, want_meta=True)
    dq, ds = roi.quantize_rows(Wm)
    pq, ps = roi.quantize_rows(vals.view(rows, cols // 2))
    assert torch.equal(ds, ps)  # the zeros of the mask change no maximum
    assert np.array_equal(dq.cpu().numpy(),
                          expand(pq.cpu().numpy(), idx.cpu().numpy(), cols))
    for tokens in (1, 16, 40, 200):
        xq, xs = roi.quantize_rows(torch.randn(tokens, cols, device="cuda").bfloat16())
        assert torch.equal(roi.linear_i8(xq, xs, dq, ds),
                           roi.linear_i8(xq, xs, pq, ps, meta=meta))


def train_step(x, gy, W, logits, n, m, seed, step):
    """One step of a masked layer with 8-bit operands and checkpoint."""
    Wm, _, _ = roi.mask_fwd(W, logits, n, m, 0.5, 1.0, seed, step, want_idx=False)
    wq, ws = roi.quantize_rows(Wm)
    xq, xs = roi.quantize_rows(x)
    y = roi.linear_i8(xq, xs, wq, ws)
    gx = roi.linear_i8_grad_input(gy, wq, ws)
    gw = roi.linear_i8_grad_weight(gy, xq, xs)
    d = roi.mask_bwd(gw, W, logits, n, m, 0.5, 1.0, seed, step)
    return y, gx, gw, d, (xq, xs, wq, ws)


@gpu
@pytest.mark.parametrize("n,m", [(2, 4), (4, 8), (8, 16)])
def test_masked_layer_step(n, m):
    """A training step of one masked layer: every output from the ones before
    it, and dL/dlogits against the oracle's from the same gradient."""
    import oracle
    import torch
    from paper_2608_23048_amd import workloads as wl
    from tests.gpu_helpers import ATOL, RTOL
    tokens, rows, cols = 150, 48, 96
    W, logits, _ = wl.small_case(rows, cols, 9, device="cuda")
    x = torch.randn(tokens, cols, device="cuda").bfloat16()
    gy = (torch.randn(tokens, rows, device="cuda") * 1e-3).bfloat16()
    y, gx, gw, d, (xq, xs, wq, ws) = train_step(x, gy, W, logits, n, m, 4, 2)
    h = lambda t: t.cpu().numpy()  # noqa: E731
    assert np.array_equal(bf16_bits(y),
                          bf16_rne_bits(linear_ref(h(xq), h(xs), h(wq), h(ws))))
    g = f32(gy.float())
    assert_grad(f32(gx.float()), g.T, h(wq), h(ws), "grad_x")
    assert_grad(f32(gw.float()), g, h(xq), h(xs), "grad_w")
    ref = oracle.mask_bwd(bf16_bits(gw).reshape(-1), bf16_bits(W).reshape(-1), h(logits), n, m,
                          0.5, 1.0, 4, 2, 0)
    err = np.abs(h(d).astype(np.float64).reshape(-1) - ref)
    assert np.all(err <= ATOL + RTOL * np.abs(ref))


@gpu
@pytest.mark.parametrize("tokens,rows,cols", [(200, 136, 272), (2000, 256, 1024)])
def test_step_in_a_graph_and_on_a_stream(tokens, rows, cols):
    """The step captured once and replayed on new inputs, with eager work
    between the replays, and on a stream of its own: the eager bits each time.
    The second size cuts its sums (a workspace in every gradient)."""
    import torch
    from paper_2608_23048_amd import workloads as wl
    assert tokens == 200 or roi.linear_i8_grad_weight_workspace(tokens, rows, cols) > 0
    W, logits, _ = wl.small_case(rows, cols, 1, device="cuda")
    x = torch.randn(tokens, cols, device="cuda").bfloat16()
    gy = torch.randn(tokens, rows, device="cuda").bfloat16()
    train_step(x, gy, W, logits, 2, 4, 0, 0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = train_step(x, gy, W, logits, 2, 4, 0, 0)[:4]
    for _ in range(4):
        x.copy_(torch.randn(tokens, cols, device="cuda"))
        gy.copy_(torch.randn(tokens, rows, device="cuda"))
        graph.replay()
        want = train_step(x, gy, W, logits, 2, 4, 0, 0)[:4]
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = train_step(x, gy, W, logits, 2, 4, 0, 0)[:4]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@gpu
def test_two_graphs_of_cut_sums_in_turn():
    """Two captured calls with workspaces of their own, replayed one after the
    other and on two streams at once."""
    import torch
    tokens, rows, cols = 3000, 300, 520
    data = [(torch.randn(tokens, rows, device="cuda").bfloat16(),
             *roi.quantize_rows(torch.randn(tokens, cols, device="cuda"))) for _ in range(2)]
    want = [roi.linear_i8_grad_weight(*d) for d in data]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for d in data:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(roi.linear_i8_grad_weight(*d))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for turn in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            if turn == 2:
                with torch.cuda.stream(s):
                    g.replay()
            else:
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@gpu
def test_given_workspace():
    import torch
    tokens, rows, cols = 3000, 300, 520
    gy = torch.randn(tokens, rows, device="cuda").bfloat16()
    x = roi.quantize_rows(torch.randn(tokens, cols, device="cuda"))
    w = roi.quantize_rows(torch.randn(rows, cols, device="cuda"))
    for fn, need, args in (
            (roi.linear_i8_grad_weight, roi.linear_i8_grad_weight_workspace, (gy, *x)),
            (roi.linear_i8_grad_input, roi.linear_i8_grad_input_workspace, (gy, *w)),
            (roi.linear_i8, roi.linear_i8_workspace, (*x, *w))):
        n = need(tokens, rows, cols)
        work = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")  # NaN as fp32
        assert torch.equal(fn(*args, workspace=work[:n] if n else None), fn(*args))
        assert (work[n:] == 255).all()
        if n:
            with pytest.raises(roi.RoiError, match="workspace"):
                fn(*args, workspace=work[:n - 16])
    assert roi.linear_i8_grad_weight_workspace(tokens, rows, cols) > 0
    with pytest.raises(roi.RoiError):
        roi.linear_i8_workspace(-1, 4, 4)


@gpu
def test_past_32_bits():
    """Rows whose elements lie past 2^32, through every operator: checked on the
    last rows."""
    import torch
    tokens, cols, rows = 67000, 65536, 24     # 4.4e9 elements
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(tokens, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    xq, xs = roi.quantize_rows(x)
    tail = x[-3:].clone()
    tq, ts = roi.quantize_rows(tail)
    assert torch.equal(xq[-3:], tq) and torch.equal(xs[-3:], ts)
    roi.dequantize_rows(xq, xs, out=x)
    assert torch.equal(x[-3:], roi.dequantize_rows(tq, ts))
    del x
    wq, ws = roi.quantize_rows(torch.empty(rows, cols, device="cuda").normal_(generator=g))
    y = roi.linear_i8(xq, xs, wq, ws)
    assert torch.equal(y[-3:], roi.linear_i8(tq, ts, wq, ws))
    gy = torch.zeros(tokens, rows, dtype=torch.bfloat16, device="cuda")
    gy[-3:].normal_(generator=g)
    gw = roi.linear_i8_grad_weight(gy, xq, xs)
    h = lambda t: t.cpu().numpy()  # noqa: E731
    assert_grad(f32(gw.float()), f32(gy[-3:].float()), h(tq), h(ts), "grad_w")
    gx = roi.linear_i8_grad_input(gy, wq, ws)
    assert torch.equal(gx[-3:], roi.linear_i8_grad_input(gy[-3:].clone(), wq, ws))
    assert (gx[:-3] == 0).all()
