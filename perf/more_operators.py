"""Cases of the training step in 8-bit floats: operands with one power-of-two
scale for each block of 128 values, their product and its gradients, and the
AdamW step over many tensors with moments in 8 bits or in 32.

A case is a dict of plain values:
  op "checkpoint": quantize_blocks of x, then dequantize_blocks
     "weight":     quantize_blocks in 128 x 128 blocks, with the transposed copy
     "linear":     quantize_blocks of the tokens, then linear_f8
     "backward":   quantize_blocks of dL/dy with its transposed copy, then
                   linear_f8_grad_input and linear_f8_grad_weight
     "adamw":      adamw_grouped over a list of tensors
  tokens, rows, cols   x [tokens, cols], weight [rows, cols]
  dtype     "bf16" or "fp32": x and its restored form ("checkpoint")
  format    "e4m3" or "e5m2": what x or dL/dy is rounded to
  bias      a bf16 bias is added
  padded    how many of the tokens, at the end, are padding: all zeros
  bits      8 or 32: the moments of "adamw"
  grad      "fp32" or "bf16": its gradients
  layers, hidden, kv, ffn   its tensors: those of a decoder stack
  count, numel              its tensors otherwise: so many, around that size

A block's scale is 2^(E - 127), with a the largest magnitude of the block and E
its biased exponent, one more where its fraction is over 3/4, less 8 (e4m3) or 15
(e5m2), at least 1; the values are x 2^(127 - E) rounded to nearest, ties to even.
The 8-bit moments are m and the root of v in e4m3 with such scales over 128
consecutive values, rounded up with the chance that their distance says: from the
bits of Philox4x32-10 words of (seed, step, element).

Activations are normal with a spread of token magnitudes and a few large
channels, as the inputs of a decoder's linear layers are; weights are 2:4-masked
N(0, 0.02^2), upstream gradients N(0, 1e-3^2) with a spread over tokens.
"""
from __future__ import annotations

import torch

own = False

BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LR, BETAS, EPS, DECAY, STEP = 1e-3, (0.9, 0.95), 1e-8, 0.05, 100
NOISE_SEED = 0x5EED0123456789AB


def listed():
    return [
        # Activations of a ragged batch of odd width, kept in 8 bits and restored.
        {"name": "checkpoint-odd-77x4865-fp32", "op": "checkpoint", "tokens": 77, "cols": 4865,
         "dtype": "fp32", "format": "e4m3", "padded": 0},
        # The widest activation of a 7B-class layer (the input of its down
        # projection) over a micro-batch, with padding at the end.
        {"name": "checkpoint-8192x18944", "op": "checkpoint", "tokens": 8192, "cols": 18944,
         "dtype": "bf16", "format": "e5m2", "padded": 300},
        # The masked up projection of a 7B-class layer, once a step: what the
        # forward and the input's gradient read.
        {"name": "weight-18944x3584", "op": "weight", "rows": 18944, "cols": 3584},
        # One token through the smallest layer: launches.
        {"name": "decode-1x896x896", "op": "linear", "tokens": 1, "rows": 896, "cols": 896,
         "format": "e4m3", "bias": True, "padded": 0},
        # A batch of 16 sequences decoding through a 7B-class down projection.
        {"name": "decode-16x3584x18944", "op": "linear", "tokens": 16, "rows": 3584,
         "cols": 18944, "format": "e4m3", "bias": False, "padded": 0},
        # A short ragged prompt through a 0.5B-class layer.
        {"name": "prefill-333x4864x896", "op": "linear", "tokens": 333, "rows": 4864, "cols": 896,
         "format": "e4m3", "bias": True, "padded": 0},
        # The forward of a micro-batch, or a long prompt, at 7B size.
        {"name": "prefill-8192x18944x3584", "op": "linear", "tokens": 8192, "rows": 18944,
         "cols": 3584, "format": "e4m3", "bias": False, "padded": 300},
        # Both gradients of a short ragged batch, a sum over an odd number of tokens.
        {"name": "backward-333x4864x896", "op": "backward", "tokens": 333, "rows": 4864,
         "cols": 896, "format": "e4m3", "padded": 0},
        # Both gradients of a 7B-class down projection over a micro-batch.
        {"name": "backward-8192x3584x18944", "op": "backward", "tokens": 8192, "rows": 3584,
         "cols": 18944, "format": "e5m2", "padded": 300},
        # The logits of one small layer, fp32 moments: launches.
        {"name": "adamw32-1x802816", "op": "adamw", "bits": 32, "grad": "fp32", "count": 1,
         "numel": 802816},
        # Many small tensors of odd sizes (biases, norms, adapters), bf16 gradients.
        {"name": "adamw8-61x5001-bf16", "op": "adamw", "bits": 8, "grad": "bf16", "count": 61,
         "numel": 5001},
        # The logits of a whole 0.5B-class stack, one per weight.
        {"name": "adamw8-stack-24x896", "op": "adamw", "bits": 8, "grad": "fp32", "layers": 24,
         "hidden": 896, "kv": 128, "ffn": 4864},
    ]


def _size(rng, lo, hi):
    """A size between 2^lo and 2^hi: odd, or a multiple of 4, 32 or 128."""
    n = 2.0 ** rng.uniform(lo, hi)
    unit = rng.choice([1, 1, 4, 32, 128, 128])
    return max(1, round(n / unit)) * unit if n >= unit else max(1, round(n))


def draw(rng):
    op = rng.choice(["checkpoint", "weight", "linear", "linear", "linear", "backward", "backward",
                     "adamw", "adamw"])
    if op == "adamw":
        count = _size(rng, 0, 7)
        # no drawn case costs more than the largest listed one
        return {"op": op, "bits": rng.choice([8, 8, 32]), "grad": rng.choice(["fp32", "bf16"]),
                "count": count, "numel": min(_size(rng, 0, 24), 180_000_000 // count)}
    cols = _size(rng, 6, 14.2)
    if op == "weight":
        return {"op": op, "rows": _size(rng, 6, 14.2), "cols": cols}
    c = {"op": op, "tokens": _size(rng, 0, 13), "cols": cols,
         "format": rng.choice(["e4m3", "e4m3", "e5m2"])}
    if op == "checkpoint":
        c["dtype"] = rng.choice(["bf16", "bf16", "fp32"])
    else:
        rows = c["rows"] = _size(rng, 6, 14.2)
        if op == "linear":
            c["bias"] = rng.random() < 0.3
        c["tokens"] = max(1, min(c["tokens"], int(5.5e11 / (rows * cols))))
    c["padded"] = rng.choice([0, 0, c["tokens"] // 10])
    return c


# ------------------------------------------------------------------- inputs
def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _words(n):
    """Scale bytes of a row of n values: whole words."""
    return (_blocks(n) + 3) // 4 * 4


def _sizes(case):
    if "layers" in case:
        h, kv, f = case["hidden"], case["kv"], case["ffn"]
        return [h * h, kv * h, kv * h, h * h, f * h, f * h, h * f] * case["layers"]
    n = case["numel"]
    return [max(1, n * (3 + 7 * i % 5) // 5 - i % 3) if i else n for i in range(case["count"])]


def _activations(case, g, dev):
    t, k = case["tokens"], case["cols"]
    x = torch.randn(t, k, generator=g, device=dev)
    x *= torch.exp(0.5 * torch.randn(t, 1, generator=g, device=dev))
    x *= 1 + 12 * (torch.rand(1, k, generator=g, device=dev) < 0.005)
    if case["padded"]:
        x[t - case["padded"]:] = 0
    return x


def _masked_weight(case, g, dev):
    r, k = case["rows"], case["cols"]
    w = torch.randn(r, k, generator=g, device=dev).mul_(0.02)
    keys = torch.rand(r, k // 4, 4, generator=g, device=dev)
    least = keys.topk(2, dim=2).values[..., 1:]
    w[:, : k // 4 * 4] *= (keys >= least).view(r, k // 4 * 4)
    return w.bfloat16()


def _strided(q):
    """q with rows that start at multiples of 16 bytes, zeros behind each."""
    r, k = q.shape
    room = torch.zeros(r, (k + 15) // 16 * 16, dtype=torch.uint8, device=q.device)
    room[:, :k] = q.view(torch.uint8)
    return room.view(q.dtype)[:, :k]


def _kept_scales(e, cols):
    """Scale bytes as they are kept: rows of whole words, 127 behind the last."""
    room = torch.full((e.shape[0], _words(cols)), 127, dtype=torch.uint8, device=e.device)
    room[:, : e.shape[1]] = e.to(torch.uint8)
    return room.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op == "adamw":
        return _prepare_adamw(case, st, g, dev)
    if op in ("checkpoint", "linear"):
        x = _activations(case, g, dev)
        st["x"] = x if case.get("dtype") == "fp32" else x.bfloat16()
    if op == "weight":
        st["x"] = _masked_weight(case, g, dev)
    if op in ("linear", "backward"):
        # held across steps: the weight, or its transposed copy, in 8 bits
        w = _masked_weight(case, g, dev).float()
        if op == "backward":
            w = w.t().contiguous()
        q, e = _quantize(w, "e4m3", True)
        st["wq"], st["ws"] = _strided(q), _kept_scales(e, w.shape[1])
    if op == "linear":
        st["bias"] = (torch.randn(case["rows"], generator=g, device=dev).mul_(0.1).bfloat16()
                      if case["bias"] else None)
    if op == "backward":
        # the forward's checkpoint: the tokens, transposed, blocks along the tokens
        q, e = _quantize(_activations(case, g, dev).bfloat16().float().t().contiguous(), "e4m3",
                         False)
        st["xq"], st["xs"] = _strided(q), _kept_scales(e, case["tokens"])
        gy = torch.randn(case["tokens"], case["rows"], generator=g, device=dev).mul_(1e-3)
        gy *= torch.exp(0.5 * torch.randn(case["tokens"], 1, generator=g, device=dev))
        if case["padded"]:
            gy[case["tokens"] - case["padded"]:] = 0
        st["gy"] = gy.bfloat16()
    return st


def _prepare_adamw(case, st, g, dev):
    """The tensors lie in slabs, each from a multiple of 2048 values on."""
    sizes = _sizes(case)
    starts, offsets, at, index = [], [], 0, 0
    for n in sizes:
        starts.append(at)
        offsets.append(index)
        at += (n + 2047) // 2048 * 2048
        index += (n + 3) // 4 * 4
    st["offsets"] = offsets
    live = torch.zeros(at + 1, dtype=torch.int32, device=dev)
    first = torch.tensor(starts, device=dev)
    live[first] += 1
    live[first + torch.tensor(sizes, device=dev)] -= 1
    live = live.cumsum(0, dtype=torch.int32)[:at] > 0
    # the global index of each block's first element
    owner = torch.searchsorted(first, torch.arange(0, at, BLOCK, device=dev), right=True) - 1
    st["first"] = (torch.arange(0, at, BLOCK, device=dev) - first[owner]
                   + torch.tensor(offsets, device=dev)[owner])
    spread = torch.exp(torch.randn(at, generator=g, device=dev))
    grad = torch.randn(at, generator=g, device=dev) * spread * live * 1e-3
    mom = torch.randn(at, generator=g, device=dev) * spread * live * 3e-4
    root = torch.rand(at, generator=g, device=dev).add_(0.2) * spread * live * 1e-3
    st["param"] = torch.randn(at, generator=g, device=dev) * live
    st["grad"] = grad.to(DTYPES[case["grad"]])
    if case["bits"] == 32:
        st["exp_avg"], st["exp_avg_sq"] = mom, root * root
    else:
        for name, x in (("mom", mom), ("root", root)):
            q, e = _quantize(x.view(1, at), "e4m3", False)
            st[name], st[name + "_scale"] = q.view(at), _bytes(e).view(-1)
    st["tensors"] = []
    for n, a in zip(sizes, starts):
        s, t = slice(a, a + n), slice(a // BLOCK, a // BLOCK + _words(n))
        moments = ((st["exp_avg"][s], st["exp_avg_sq"][s]) if case["bits"] == 32 else
                   ((st["mom"][s], st["mom_scale"][t]), (st["root"][s], st["root_scale"][t])))
        st["tensors"].append((st["param"][s], st["grad"][s], *moments))
    return st


def _bytes(e):
    return e.to(torch.uint8).view(torch.float8_e8m0fnu)


# ---------------------------------------------------------------------- run
def _exponent(a, fmt):
    """Scale bytes of blocks whose largest magnitudes are a (fp32)."""
    return (((a.view(torch.int32) + 0x1FFFFF) >> 23) - (8 if fmt == "e4m3" else 15)).clamp_min(1)


def _power(e):
    """2^(e - 127) in fp32, for e from 1 to 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _spread(e, rows, cols, square):
    """The blocks' values at each of their elements."""
    e = e.repeat_interleave(BLOCK, dim=1)[:, :cols]
    return e.repeat_interleave(BLOCK, dim=0)[:rows] if square else e


def _quantize(x, fmt, square):
    """(8-bit values, scale bytes [blocks of rows, blocks of cols]) of x, fp32."""
    r, k = x.shape
    room = torch.zeros(_blocks(r) * BLOCK if square else r, _blocks(k) * BLOCK, device=x.device)
    room[:r, :k] = x.abs()
    if square:
        a = room.view(_blocks(r), BLOCK, _blocks(k), BLOCK).amax(dim=(1, 3))
    else:
        a = room.view(r, _blocks(k), BLOCK).amax(dim=2)
    e = _exponent(a, fmt)
    return (x * _spread(_power(254 - e), r, k, square)).to(FORMATS[fmt]), e


def _restore(q, e, square=False):
    """fp32 values; e: scale bytes, or the scales as they are kept."""
    r, k = q.shape
    if e.dtype is torch.float8_e8m0fnu:
        e = e.view(torch.uint8)
    return q.float() * _spread(_power(e[:, : _blocks(k)]), r, k, square)


def _philox(index, seed, step):
    """The words of elements index .. index + 3 (index a multiple of 4): four
    tensors of 32-bit values held in 64."""
    low = 0xFFFFFFFF
    block = index >> 2
    a, b = block & low, block >> 32
    c, d = torch.full_like(a, step & low), torch.full_like(a, step >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57  # modulo 2^64: both words are whole
        a, b, c, d = (q >> 32) & low ^ b ^ k0, q & low, (p >> 32) & low ^ d ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return a, b, c, d


def _round_by(t, bits):
    """t >= 0 (fp32, at most 448) to e4m3, up with the chance of 20 random bits."""
    normal = ((t.view(torch.int32) + bits) & ~0xFFFFF).view(torch.float32)
    small = torch.floor(t.double() * 512 + bits.double() / 2 ** 20).float() / 512
    return torch.where(t >= 2.0 ** -6, normal, small)


def _plain_adamw(st):
    c1, c2 = 1 - BETAS[0] ** STEP, 1 - BETAS[1] ** STEP
    g = st["grad"].float()
    if st["case"]["bits"] == 32:
        m, v = st["exp_avg"], st["exp_avg_sq"]
    else:
        m = st["mom"].float().view(-1, BLOCK) * _power(st["mom_scale"].view(torch.uint8))[:, None]
        r = st["root"].float().view(-1, BLOCK) * _power(st["root_scale"].view(torch.uint8))[:, None]
        m, v = m.view(-1), (r * r).view(-1)
    m = m * BETAS[0] + g * (1 - BETAS[0])
    v = v * BETAS[1] + g * g * (1 - BETAS[1])
    root = v.sqrt()
    p = st["param"]
    p.copy_(p * (1 - LR * DECAY) - LR / c1 * m / (root / c2 ** 0.5 + EPS))
    if st["case"]["bits"] == 32:
        st["exp_avg"].copy_(m)
        st["exp_avg_sq"].copy_(v)
        return {k: st[k] for k in ("param", "exp_avg", "exp_avg_sq")}
    index = st["first"][:, None] + torch.arange(0, BLOCK, 4, device=p.device)
    word = torch.stack(_philox(index, NOISE_SEED, STEP), dim=-1).view(-1, BLOCK)
    for name, x, bits in (("mom", m, (word & 0xFFF) << 8), ("root", root, word >> 12)):
        x = x.view(-1, BLOCK)
        e = _exponent(x.abs().amax(dim=1), "e4m3")
        t = _round_by((x * _power(254 - e)[:, None]).abs(), bits.to(torch.int32))
        if name == "root":  # never 0 but for 0
            t = torch.where(x > 0, t.clamp_min(2.0 ** -9), t)
        st[name].copy_(torch.copysign(t, x).to(torch.float8_e4m3fn).view(-1))
        st[name + "_scale"].copy_(_bytes(e))
    return {k: st[k] for k in ("param", "mom", "mom_scale", "root", "root_scale")}


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "adamw":
        return _plain_adamw(st)
    if op == "checkpoint":
        q, e = _quantize(st["x"].float(), case["format"], False)
        return {"q": q, "scale": _bytes(e), "x": _restore(q, e).to(DTYPES[case["dtype"]])}
    if op == "weight":
        q, e = _quantize(st["x"].float(), "e4m3", True)
        return {"q": q, "scale": _bytes(e), "qt": q.t().contiguous(),
                "scale_t": _bytes(e.t().contiguous())}
    if op == "linear":
        q, e = _quantize(st["x"].float(), case["format"], False)
        y = torch.matmul(_restore(q, e), _restore(st["wq"], st["ws"], True).t())
        if st["bias"] is not None:
            y = y + st["bias"].float()
        return y.bfloat16()
    gy = st["gy"].float()
    q, e = _quantize(gy, case["format"], False)
    gx = torch.matmul(_restore(q, e), _restore(st["wq"], st["ws"], True).t()).bfloat16()
    q, e = _quantize(gy.t().contiguous(), case["format"], False)
    gw = torch.matmul(_restore(q, e), _restore(st["xq"], st["xs"]).t()).bfloat16()
    return {"gx": gx, "gw": gw}


def run(st):
    if not own:
        return _plain(st)
    import paper_2608_23048_amd as roi
    case = st["case"]
    op = case["op"]
    if op == "adamw":
        if "plan" not in st:  # once, as a training program keeps its optimizer
            st["plan"] = roi.adamw_plan(st["tensors"], offsets=st["offsets"])
        roi.adamw_grouped(st["plan"], roi.adamw_params(LR, BETAS, EPS, DECAY, STEP),
                          seed=NOISE_SEED, step=STEP)
        names = (("param", "mom", "mom_scale", "root", "root_scale") if case["bits"] == 8
                 else ("param", "exp_avg", "exp_avg_sq"))
        return {k: st[k] for k in names}
    if op == "checkpoint":
        q, s = roi.quantize_blocks(st["x"], dtype=FORMATS[case["format"]])
        return {"q": q, "scale": s[:, : _blocks(case["cols"])],
                "x": roi.dequantize_blocks(q, s, dtype=DTYPES[case["dtype"]])}
    if op == "weight":
        q, s, qt, t = roi.quantize_blocks(st["x"], square=True, transposed=True)
        return {"q": q, "scale": s[:, : _blocks(case["cols"])], "qt": qt,
                "scale_t": t[:, : _blocks(case["rows"])]}
    if op == "linear":
        q, s = roi.quantize_blocks(st["x"], dtype=FORMATS[case["format"]])
        return roi.linear_f8(q, s, st["wq"], st["ws"], bias=st["bias"])
    q, s, qt, t = roi.quantize_blocks(st["gy"], transposed=True, dtype=FORMATS[case["format"]])
    return {"gx": roi.linear_f8_grad_input(q, s, st["wq"], st["ws"]),
            "gw": roi.linear_f8_grad_weight(qt, t, st["xq"], st["xs"])}


# --------------------------------------------------------- work and reference
def work(case):
    op = case["op"]
    if op == "adamw":
        n = sum(_sizes(case))
        moments = 16 * n if case["bits"] == 32 else 4 * n + 4 * sum(map(_blocks, _sizes(case)))
        return {"bytes": n * (8 + (4 if case["grad"] == "fp32" else 2)) + moments, "flops": 14 * n}
    k = case["cols"]
    if op == "checkpoint":
        # saved in the forward, restored in the backward
        t, size = case["tokens"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": t * k * (2 * size + 2) + 2 * t * _blocks(k), "flops": 4 * t * k}
    r = case["rows"]
    if op == "weight":
        return {"bytes": 4 * r * k + 2 * _blocks(r) * _blocks(k), "flops": 4 * r * k}
    t = case["tokens"]
    if op == "linear":
        return {"bytes": 2 * t * k + r * k + _blocks(r) * _blocks(k) + 2 * t * r
                + (2 * r if case["bias"] else 0), "flops": 2 * t * r * k}
    return {"bytes": 2 * t * r + r * k + t * k + k * _blocks(t) + _blocks(r) * _blocks(k)
            + 2 * t * k + 2 * r * k, "flops": 4 * t * r * k}


def _two_to(power):
    """2^power in 64 bits, exactly."""
    return (power.to(torch.int64) + 1023 << 52).view(torch.float64)


def exact(case, seed):
    """From the definitions, in 64 bits."""
    st = prepare(case, seed)
    op = case["op"]
    wide = torch.float64

    def scale_of(top, fmt):
        """2^(E - 127) from the largest magnitudes."""
        half, power = torch.frexp(top)  # top = half 2^power, half in [1/2, 1)
        power = power - 1 + (half * 2 > 1.75).to(power.dtype)
        power = torch.where(top > 0, power - {"e4m3": 8, "e5m2": 15}[fmt], torch.full_like(power, -126))
        return _two_to(power.clamp(min=-126))

    def by_block(x, square, fmt):
        """The scale at every element of x, and one for each block."""
        r, k = x.shape
        grown = torch.nn.functional.pad(x.abs(), (0, -k % BLOCK, 0, -r % BLOCK if square else 0))
        high = BLOCK if square else 1
        cut = grown.unfold(0, high, high).unfold(1, BLOCK, BLOCK)
        s = scale_of(cut.amax(dim=(2, 3)), fmt)
        rows = torch.arange(r, device=x.device) // high
        cols = torch.arange(k, device=x.device) // BLOCK
        return s[rows][:, cols], s

    def nearest(t, fmt):
        """t to the nearest of the format's values, ties to even."""
        digits, lowest = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
        step = _two_to((torch.frexp(t)[1] - 1).clamp(min=lowest) - digits)
        return torch.round(t / step) * step

    def held(x, fmt, square):
        s, small = by_block(x, square, fmt)
        return nearest(x / s, fmt), s, small

    def kept(q, s, square):
        r, k = q.shape
        scale = _two_to(s.view(torch.uint8).to(torch.int64) - 127)
        rows = torch.arange(r, device=q.device) // (BLOCK if square else 1)
        cols = torch.arange(k, device=q.device) // BLOCK
        return q.to(wide) * scale[rows][:, cols]

    if op == "adamw":
        return _exact_adamw(st, scale_of)
    if op in ("checkpoint", "weight"):
        q, s, small = held(st["x"].to(wide), case.get("format", "e4m3"), op == "weight")
        if op == "weight":
            return {"q": q, "scale": small, "qt": q.t(), "scale_t": small.t()}
        return {"q": q, "scale": small, "x": q * s}
    if op == "linear":
        q, s, _ = held(st["x"].to(wide), case["format"], False)
        y = torch.mm(q * s, kept(st["wq"], st["ws"], True).t().contiguous())
        return y if st["bias"] is None else y + st["bias"].to(wide)
    gy = st["gy"].to(wide)
    q, s, _ = held(gy, case["format"], False)
    gx = torch.mm(q * s, kept(st["wq"], st["ws"], True).t().contiguous())
    q, s, _ = held(gy.t().contiguous(), case["format"], False)
    return {"gx": gx, "gw": torch.mm(q * s, kept(st["xq"], st["xs"], False).t().contiguous())}


def _exact_adamw(st, scale_of):
    wide = torch.float64
    one = [1 - b for b in BETAS]
    g = st["grad"].to(wide)
    eight = st["case"]["bits"] == 8
    if eight:
        at = torch.arange(g.numel(), device=g.device) // BLOCK
        m, v = (st[k].to(wide) * _two_to(st[k + "_scale"].view(torch.uint8).to(torch.int64) - 127)[at]
                for k in ("mom", "root"))
        v = v ** 2
    else:
        m, v = st["exp_avg"].to(wide), st["exp_avg_sq"].to(wide)
    m, v = BETAS[0] * m + one[0] * g, BETAS[1] * v + one[1] * g ** 2
    ahead, spread = m / (1 - BETAS[0] ** STEP), torch.sqrt(v / (1 - BETAS[1] ** STEP))
    p = st["param"].to(wide)
    p = p - LR * DECAY * p - LR * ahead / (spread + EPS)
    if not eight:
        return {"param": p, "exp_avg": m, "exp_avg_sq": v}

    # the words of all elements, from products of 16-bit halves
    def times(x, c):
        lo, hi = (x & 0xFFFF) * c, (x >> 16) * c
        hi += lo >> 16
        return hi >> 16, (hi & 0xFFFF) << 16 | lo & 0xFFFF

    block = (st["first"][:, None] + torch.arange(0, BLOCK, 4, device=g.device)) // 4
    x = [block % 2 ** 32, block // 2 ** 32, torch.full_like(block, STEP), torch.zeros_like(block)]
    key = [NOISE_SEED % 2 ** 32, NOISE_SEED // 2 ** 32]
    for _ in range(10):
        (h0, l0), (h1, l1) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    word = torch.stack(x, dim=2).reshape(-1, BLOCK)
    out = {"param": p}
    for name, y, chance in (("mom", m, (word % 2 ** 12).to(wide) / 2 ** 12),
                            ("root", torch.sqrt(v), (word // 2 ** 12).to(wide) / 2 ** 20)):
        y = y.view(-1, BLOCK)
        s = scale_of(y.abs().amax(dim=1, keepdim=True), "e4m3")
        t = y.abs() / s
        step = _two_to((torch.frexp(t)[1] - 1).clamp(min=-6) - 3)
        t = torch.floor(t / step + chance) * step
        if name == "root":
            t = torch.where(y > 0, t.clamp(min=2.0 ** -9), t)
        out[name], out[name + "_scale"] = (t * torch.sign(y)).view(-1), s.view(-1)
    return out
