"""adamw_grouped in 8 bits over the whole of fp32's range: gradients whose squares fp32 does
not hold, moments next to 2^128, and elements that are not finite among others.

The stored moments are compared byte for byte with 64-bit arithmetic: m' and sqrt(v') as
products and sums of doubles, then floor(t / u + chance) u with the chance of the
element's noise word.  The parameter's tolerance is test_f8's, of a step in fp32.
"""
from __future__ import annotations

import pytest
import torch

import paper_2608_23048_amd as roi
from tests.test_f8 import step_ref

SEED, STEP = 7, 3


def power(e):
    """2^e in 64 bits, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def held(q, s):
    n = q.numel()
    return q.double() * power(s.view(torch.uint8).long() - 127).repeat_interleave(128)[:n]


def block_most(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % 128)).view(-1, 128).amax(1)


def stepped(g, m, r, betas):
    """(values, E) of both moments after a step; NaN where the gradient or the old moment is one
    or an infinity, which E does not count."""
    b1, b2 = betas
    n = g.numel()
    g = g.double()
    word = roi.gumbel_noise((n + 3) // 4 * 4, SEED, STEP, 0, want_gumbel=False)[0][:n].long() & 0xFFFFFFFF
    root = held(*r)
    first = b1 * held(*m) + (1 - b1) * g
    second = (b2 * (root * root) + (1 - b2) * (g * g)).sqrt()
    out = []
    for x, chance in ((first, (word % 4096).double() / 4096), (second, (word // 4096).double() / 2 ** 20)):
        ok = torch.isfinite(x)
        a = torch.where(ok, x.abs(), torch.zeros_like(x))
        e = ((block_most(a).view(torch.int64) + 2 ** 50 - 1) >> 52) - 1023 + 127 - 8
        e = e.clamp_min(1)
        t = a * power(127 - e).repeat_interleave(128)[:n]
        u = power(((t.view(torch.int64) >> 52) - 1023).clamp_min(-6) - 3)
        t = torch.floor(t / u + chance) * u
        if x is second:
            t = torch.where(a > 0, t.clamp_min(2.0 ** -9), t)
        out.append((torch.where(ok, torch.copysign(t, x), torch.full_like(t, float("nan"))), e))
    return out


def same_moments(got, want):
    for (q, s), (t, e) in zip(got, want):
        assert torch.equal(s.view(torch.uint8)[: e.numel()].long(), e)
        nan = torch.isnan(t)
        assert torch.equal(torch.isnan(q.float()), nan)
        assert torch.equal(q.double()[~nan], t[~nan])


def state(n, seed, size=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda: torch.randn(n, generator=g, device="cuda")
    wide = torch.exp(2 * normal())
    return (normal(), normal() * wide * size, roi.quantize_blocks(normal() * wide * 0.3 * size),
            roi.quantize_blocks(normal().abs() * wide * size))


def check(p, grad, m, r, opt, betas):
    """One step in place; the parameter and both moments are right."""
    want = stepped(grad.float(), m, r, betas)
    h = [held(*m).cpu(), held(*r).cpu()]
    p1, _, _, ep, _ = step_ref(p.double().cpu(), grad.double().cpu(), h[0], h[1] * h[1], opt)
    roi.adamw_grouped([(p, grad, m, r)], opt, seed=SEED, step=STEP)
    same_moments((m, r), want)
    ok = torch.isfinite(p1)
    assert bool(((p.double().cpu() - p1).abs() <= ep)[ok].all())
    assert not torch.isfinite(p.cpu()[~ok]).any()


HUGE = [1e20, -3e38, 1.9e19, 5e19, 1.8e19, -1.85e19, 3.4e38, 2.0 ** 64, -2.0 ** 127]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("betas", [(0.9, 0.95), (0.0, 0.0), (0.9, 0.999)])
def test_gradients_whose_squares_pass_fp32(betas, dtype):
    n = 128 * 41 + 77
    p, grad, m, r = state(n, 5)
    for i, v in enumerate(HUGE):  # some alone in their 256 elements, some together
        grad[i * 397 + i] = v
        grad[3840 + 7 * i] = -v
    grad = grad.clamp(-3.38e38, 3.38e38).to(dtype)
    for t in range(1, 4):
        check(p, grad, m, r, roi.adamw_params(1e-3, betas, t=t), betas)
        assert bool(torch.isfinite(p).all())
        grad = grad * 0 if t == 1 else torch.randn_like(p).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("betas", [(0.9, 0.95), (0.5, 0.0), (0.0, 0.999)])
def test_moments_next_to_2_128(betas):
    """Both moments of some elements are held as 2^128, which fp32 has not."""
    n = 1000
    p, grad, m, r = state(n, 6, 1e33)
    top = torch.zeros(n, device="cuda")
    top[::51] = 3.4e38
    m, r = roi.quantize_blocks(top), roi.quantize_blocks(top)
    assert float(held(*m).max()) == float(held(*r).max()) == 2.0 ** 128
    for t in range(1, 4):
        check(p, grad, m, r, roi.adamw_params(1e-3, betas, t=t), betas)
        assert bool(torch.isfinite(p).all())


@pytest.mark.gpu
def test_what_is_not_finite_changes_no_other():
    """One such element in each 256: the others' moments are those of 64 bits."""
    n = 1 << 24
    p, grad, m, r = state(n, 8)
    at = torch.arange(0, n, 256, device="cuda") + torch.arange(n // 256, device="cuda") % 256
    bad = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda")
    grad[at] = bad[torch.arange(at.numel(), device="cuda") % 3]
    clean = grad.clone()
    clean[at] = 0
    opt = roi.adamw_params(1e-3, (0.9, 0.95), t=9)
    for dirty in (grad, clean):  # the second step begins with NaN among the moments
        want = stepped(dirty, m, r, (0.9, 0.95))
        a, b = p.clone(), p.clone()
        again = tuple(tuple(t.clone() for t in k) for k in (m, r))
        roi.adamw_grouped([(a, dirty, m, r)], opt, seed=SEED, step=STEP)
        roi.adamw_grouped([(b, clean, *again)], opt, seed=SEED, step=STEP)
        same_moments((m, r), want)
        a[at] = b[at] = 0
        assert torch.equal(a, b)
