"""Cases of the 8-bit linear layer around a masked weight: rows of activations
quantized to int8 (the product's operand and the backward's checkpoint), the
integer product with dense or 2:4-compressed weights, and the two gradients
that read 8-bit operands.

A case is a dict of plain values:
  op       "checkpoint":  quantize_rows, then dequantize_rows
           "linear":      quantize_rows of the tokens, then linear_i8
           "grad_weight": linear_i8_grad_weight from a saved checkpoint
           "grad_input":  linear_i8_grad_input
  tokens, rows, cols       x [tokens, cols], weight [rows, cols]
  dtype    "bf16" or "fp32": x and its restored form ("checkpoint"), or the
           output ("linear")
  packed   the weight is 2:4-compressed (values and metadata words)
  bias     a bf16 bias is added
  padded   how many of the tokens, at the end, are padding: all zeros

The quantizer is a fixed sequence of fp32 operations per row, so that its
integers are reproducible: scale = max(fl(amax / 127), 2^-126),
inv = fl(127 / amax) (2^126 at that floor), q = rint(fl(x inv)).

Activations are normal with a spread of token magnitudes and a few large
channels, as the inputs of a decoder's linear layers are; weights are
N(0, 0.02^2), upstream gradients N(0, 1e-3^2) with a spread over tokens.
"""
from __future__ import annotations

import torch

own = False

FLOOR = 2.0 ** -126   # the smallest scale of a row
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # Activations of a ragged batch of odd width, kept in 8 bits and restored.
        {"name": "checkpoint-odd-77x4865-fp32", "op": "checkpoint", "tokens": 77, "cols": 4865,
         "dtype": "fp32", "padded": 0},
        # The widest activation of a 7B-class layer (the input of its down
        # projection) over a micro-batch, with padding at the end.
        {"name": "checkpoint-8192x18944", "op": "checkpoint", "tokens": 8192, "cols": 18944,
         "dtype": "bf16", "padded": 300},
        # One token through the smallest exported layer: launches.
        {"name": "decode-1x896x896-2of4", "op": "linear", "tokens": 1, "rows": 896, "cols": 896,
         "dtype": "bf16", "packed": True, "bias": True, "padded": 0},
        # One token through the up projection of a 7B-class layer, 2:4 weights.
        {"name": "decode-1x18944x3584-2of4", "op": "linear", "tokens": 1, "rows": 18944,
         "cols": 3584, "dtype": "bf16", "packed": True, "bias": False, "padded": 0},
        # A batch of 16 sequences decoding through its down projection, dense.
        {"name": "decode-16x3584x18944", "op": "linear", "tokens": 16, "rows": 3584,
         "cols": 18944, "dtype": "bf16", "packed": False, "bias": False, "padded": 0},
        # A short ragged prompt through a 0.5B-class layer, fp32 results.
        {"name": "prefill-333x4864x896-fp32", "op": "linear", "tokens": 333, "rows": 4864,
         "cols": 896, "dtype": "fp32", "packed": False, "bias": True, "padded": 0},
        # The forward of a micro-batch, or a long prompt, at 7B size.
        {"name": "prefill-8192x18944x3584", "op": "linear", "tokens": 8192, "rows": 18944,
         "cols": 3584, "dtype": "bf16", "packed": False, "bias": False, "padded": 300},
        # A prompt through the exported 2:4 down projection.
        {"name": "prefill-4096x3584x18944-2of4", "op": "linear", "tokens": 4096, "rows": 3584,
         "cols": 18944, "dtype": "bf16", "packed": True, "bias": False, "padded": 0},
        # dL/dW_masked of a small layer: few outputs, a long sum over tokens.
        {"name": "grad-weight-4096x896x896", "op": "grad_weight", "tokens": 4096, "rows": 896,
         "cols": 896, "padded": 100},
        # dL/dW_masked of the largest layer over a micro-batch.
        {"name": "grad-weight-8192x18944x3584", "op": "grad_weight", "tokens": 8192,
         "rows": 18944, "cols": 3584, "padded": 300},
        # dL/dx of a short ragged batch.
        {"name": "grad-input-333x4864x896", "op": "grad_input", "tokens": 333, "rows": 4864,
         "cols": 896, "padded": 0},
        # dL/dx of the down projection over a micro-batch.
        {"name": "grad-input-8192x3584x18944", "op": "grad_input", "tokens": 8192, "rows": 3584,
         "cols": 18944, "padded": 300},
    ]


def _size(rng, lo, hi):
    """A size between 2^lo and 2^hi: odd, or a multiple of 4, 32 or 128."""
    n = 2.0 ** rng.uniform(lo, hi)
    unit = rng.choice([1, 1, 4, 32, 128, 128])
    return max(1, round(n / unit)) * unit if n >= unit else max(1, round(n))


def draw(rng):
    op = rng.choice(["checkpoint", "linear", "linear", "linear", "grad_weight", "grad_weight",
                     "grad_input"])
    tokens = _size(rng, 0, 13)
    cols = _size(rng, 6, 14.2)
    c = {"op": op, "tokens": tokens}
    if op == "checkpoint":
        c.update({"cols": cols, "dtype": rng.choice(["bf16", "bf16", "fp32"])})
    else:
        rows = _size(rng, 6, 14.2)
        if op == "linear":
            packed = rng.random() < 0.5
            if packed:  # the metadata words of a row are whole
                cols = max(32, cols // 32 * 32)
            c.update({"dtype": rng.choice(["bf16", "bf16", "fp32"]), "packed": packed,
                      "bias": rng.random() < 0.3})
        # no drawn case costs more than the largest listed one
        tokens = c["tokens"] = max(1, min(tokens, int(5.5e11 / (rows * cols))))
        c.update({"rows": rows, "cols": cols})
    c["padded"] = rng.choice([0, 0, tokens // 10])
    return c


# ------------------------------------------------------------------- inputs
def _activations(case, g, dev):
    t, k = case["tokens"], case["cols"]
    x = torch.randn(t, k, generator=g, device=dev)
    x *= torch.exp(0.5 * torch.randn(t, 1, generator=g, device=dev))
    x *= 1 + 12 * (torch.rand(1, k, generator=g, device=dev) < 0.005)
    if case["padded"]:
        x[t - case["padded"]:] = 0
    return x


def _quantize(x):
    """The quantizer in elementary operations, fp32."""
    amax = x.abs().amax(dim=1)
    scale = (amax / 127).clamp_min(FLOOR)
    inv = torch.where(scale > FLOOR, 127 / amax, 1 / FLOOR)
    return torch.round(x * inv[:, None]), scale


def _weights(case, g, dev):
    """(wq, ws, meta): int8 rows with their scales; 2:4: the two kept values of
    every group of four in index order, and the metadata words."""
    r, k = case["rows"], case["cols"]
    w = torch.randn(r, k, generator=g, device=dev).mul_(0.02).bfloat16().float()
    if not case.get("packed"):
        q, s = _quantize(w)
        return q.to(torch.int8), s, None
    keys = torch.rand(r, k // 4, 4, generator=g, device=dev)
    idx = keys.topk(2, dim=2).indices.sort(dim=2).values
    kept = w.view(r, k // 4, 4).gather(2, idx).reshape(r, k // 2)
    nib = (idx[..., 0] | (idx[..., 1] << 2)).view(-1, 8)
    word = (nib << (4 * torch.arange(8, device=dev))).sum(dim=1)
    q, s = _quantize(kept)
    return q.to(torch.int8), s, torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op in ("checkpoint", "linear"):
        x = _activations(case, g, dev)
        st["x"] = x if op == "checkpoint" and case["dtype"] == "fp32" else x.bfloat16()
    if op == "grad_weight":
        q, st["xs"] = _quantize(_activations(case, g, dev).bfloat16().float())
        st["xq"] = q.to(torch.int8)
    if op in ("linear", "grad_input"):
        st["wq"], st["ws"], st["meta"] = _weights(case, g, dev)
    if op == "linear":
        st["bias"] = (torch.randn(case["rows"], generator=g, device=dev).mul_(0.1).bfloat16()
                      if case["bias"] else None)
    if op in ("grad_weight", "grad_input"):
        gy = torch.randn(case["tokens"], case["rows"], generator=g, device=dev).mul_(1e-3)
        gy *= torch.exp(0.5 * torch.randn(case["tokens"], 1, generator=g, device=dev))
        if case["padded"]:
            gy[case["tokens"] - case["padded"]:] = 0
        st["gy"] = gy.bfloat16()
    return st


# ---------------------------------------------------------------------- run
def _expand(wq, meta):
    """The dense fp32 rows of 2:4-compressed ones."""
    r, half = wq.shape
    shift = 4 * torch.arange(8, device=wq.device, dtype=torch.int32)
    nib = (meta[:, None] >> shift) & 15
    idx = torch.stack([nib & 3, nib >> 2], dim=-1).view(r, half // 2, 2).long()
    dense = torch.zeros(r, half // 2, 4, device=wq.device)
    return dense.scatter_(2, idx, wq.float().view(r, half // 2, 2)).view(r, 2 * half)


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "checkpoint":
        q, s = _quantize(st["x"].float())
        return (q * s[:, None]).to(DTYPES[case["dtype"]])
    if op == "linear":
        q, s = _quantize(st["x"].float())
        w = st["wq"].float() if st["meta"] is None else _expand(st["wq"], st["meta"])
        y = torch.matmul(q, w.t()) * st["ws"] * s[:, None]
        if st["bias"] is not None:
            y = y + st["bias"].float()
        return y.to(DTYPES[case["dtype"]])
    gy = st["gy"].float()
    if op == "grad_weight":
        return torch.matmul(gy.t(), st["xq"].float() * st["xs"][:, None]).bfloat16()
    return torch.matmul(gy, st["wq"].float() * st["ws"][:, None]).bfloat16()


def run(st):
    if not own:
        return _plain(st)
    import paper_2608_23048_amd as roi
    case = st["case"]
    op = case["op"]
    if op == "checkpoint":
        q, s = roi.quantize_rows(st["x"])
        return roi.dequantize_rows(q, s, dtype=DTYPES[case["dtype"]])
    if op == "linear":
        q, s = roi.quantize_rows(st["x"])
        return roi.linear_i8(q, s, st["wq"], st["ws"], meta=st["meta"], bias=st["bias"],
                             dtype=DTYPES[case["dtype"]])
    if op == "grad_weight":
        return roi.linear_i8_grad_weight(st["gy"], st["xq"], st["xs"])
    return roi.linear_i8_grad_input(st["gy"], st["wq"], st["ws"])


# --------------------------------------------------------- work and reference
def work(case):
    t, k = case["tokens"], case["cols"]
    if case["op"] == "checkpoint":
        # saved in the forward, restored in the backward: the 8-bit rows and
        # their scales are written once and read once
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": t * k * (2 * size + 2) + 8 * t, "flops": 4 * t * k}
    r = case["rows"]
    if case["op"] == "linear":
        packed = case["packed"]
        weight = r * k * 5 // 8 if packed else r * k
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * t * k + weight + 4 * r + size * t * r + (2 * r if case["bias"] else 0),
                "flops": t * r * k * (1 if packed else 2)}
    if case["op"] == "grad_weight":
        return {"bytes": 2 * t * r + t * k + 4 * t + 2 * r * k, "flops": 2 * t * r * k}
    return {"bytes": 2 * t * r + r * k + 4 * r + 2 * t * k, "flops": 2 * t * r * k}


def exact(case, seed):
    """From the definitions: the integers by the quantizer's fp32 sequence, all
    sums and products in 64 bits."""
    st = prepare(case, seed)
    op = case["op"]
    wide = torch.float64

    def ints(x):
        a = x.float()
        top = a.abs().max(dim=1, keepdim=True).values
        low = top / 127 < FLOOR
        inv = torch.where(low, torch.full_like(top, 2.0 ** 126), torch.full_like(top, 127.0) / top)
        step = torch.where(low, torch.full_like(top, FLOOR).to(wide), top.to(wide) / 127)
        return (a * inv).round().to(wide), step

    if op == "checkpoint":
        n, step = ints(st["x"])
        return n * step
    if op == "grad_weight":
        return torch.mm(st["gy"].to(wide).t().contiguous(),
                        st["xq"].to(wide) * st["xs"].to(wide).unsqueeze(1))
    w = st["wq"].to(wide)
    if st["meta"] is not None:
        r, k = case["rows"], case["cols"]
        full = torch.zeros(r * k // 4, 4, dtype=wide, device=w.device)
        words = st["meta"].to(torch.int64)
        group = torch.arange(r * k // 4, device=w.device)
        field = (words[group // 8] >> (4 * (group % 8))) & 15
        for j in (0, 1):
            full[group, (field >> (2 * j)) & 3] = w.reshape(-1, 2)[:, j]
        w = full.reshape(r, k)
    w = w * st["ws"].to(wide).unsqueeze(1)
    if op == "grad_input":
        return torch.mm(st["gy"].to(wide), w)
    n, step = ints(st["x"])
    y = torch.mm(n * step, w.t().contiguous())
    return y if st["bias"] is None else y + st["bias"].to(wide)
