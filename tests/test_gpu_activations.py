"""The activations and their slopes by themselves: a layer of one input, one output and weight 1, against the formulas in 64 bits.

Bound, relative, with u = 2^-24 and |z| <= 13.  gelu = z Phi(z) with Phi(-|z|) = Q(t) e^(-z^2 / 2), t = 1 / (1 + p |z|):  the exponent z^2 log2(e) / 2 is rounded
three times (square, constant, product), which e^() makes 1.5 z^2 u of; ex2.approx 2^-22, rcp.approx 2^-23; the denominator, ten steps of a sum of positive
size and three products about 16 u; Q itself 2^-23 in fp32, 2^-16 in 16-bit types.  Together 2^-19 + 1.5 z^2 u (fp32), 2^-15 + 1.5 z^2 u (16 bits).  For z > 0 the error
of 1 - Phi(-z) is below that.  The slope Phi + z phi has the same error of either term.  silu: the exponent is rounded twice (|z| u each), the rest is below 2^-19.
z is x exactly: 1 times a value of at most 14 bits (the lower part of an fp32 operand then has 3).  dx = slope * 1 loses the bits of that lower part that a TF32 operand drops,
2^-21, and is rounded to the type twice (as dz and as dx, the same value).
"""
import math

import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LEAST = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -25}     # what lies below may be lost


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", [hpf.ACT_GELU, hpf.ACT_SILU])
def test_value_and_slope(act, dtype):
    t = TYPES[dtype]
    x = (torch.arange(-13 * 1024, 13 * 1024 + 1, device=DEV) / 1024).to(t)[:, None].contiguous()
    rows = x.shape[0]
    one = torch.ones(1, 1, dtype=t, device=DEV)
    y, z, dx, dy = (torch.ones(rows, 1, dtype=t, device=DEV) for _ in range(4))
    size = (rows, 1, 1, 1, 1)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size, t, act), dtype=torch.uint8, device=DEV)
    hpf.linear_fwd(x, one, None, None, y, z, *size, act, scratch)
    hpf.linear_bwd(dy, z, x, one, dx, None, None, *size, act, scratch)
    torch.cuda.synchronize()
    assert torch.equal(z, x)
    v = x.double()
    u = 2.0 ** -24
    if act == hpf.ACT_GELU:
        a, b = 0.5 * torch.erfc(-v / math.sqrt(2)), v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        rel = (2.0 ** -19 if dtype == "fp32" else 2.0 ** -15) + 1.5 * v * v * u
    else:
        a = torch.sigmoid(v)
        b = v * a * torch.sigmoid(-v)
        rel = 2.0 ** -19 + 2 * v.abs() * u
    half = torch.finfo(t).eps / 2
    want = v * a
    off = (y.double() - want).abs() / (want.abs() * (rel + half) + LEAST[dtype])
    assert off.max() <= 1, (off.max().item(), v.flatten()[off.argmax()].item())
    slope = a + b
    off = (dx.double() - slope).abs() / ((a + b.abs()) * (rel + 2.0 ** -21) + half * slope.abs() + LEAST[dtype])
    assert off.max() <= 1, (off.max().item(), v.flatten()[off.argmax()].item())
