"""Sums of very many products with 16-bit results.

Bound.  The accumulator truncates: an addition of 16 products moves the sum towards zero by at most one step of fp32, 2^-23 of the sum so far, and as much
for what one instruction adds up inside.  Sums leave it after at most 512 additions and go on in registers, rounded to nearest: 2 * 512 * 2^-23 = 2^-13 of
the largest partial sum, plus 2^-24 for each of the N = K / 16 / 256 + 8 partial sums that are added up (in error the root of their number: independent
roundings to nearest; 8 standard deviations are allowed).  With operands of one sign the largest partial sum is the result itself; with random signs it is taken as
the root of the sum of squares times 5.  A rounding to the type is off by half a step, and on average over N results by half a step / sqrt(3 N): six of these
are allowed in the mean.
"""
import math

import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _bound(K):
    return 2 * 512 * 2.0 ** -23 + 8 * math.sqrt(K / 4096 + 8) * 2.0 ** -24


def _operand(g, rows, cols, scale, one_sign, t):
    v = torch.rand(rows, cols, generator=g, device=DEV) + 0.5 if one_sign else torch.randn(rows, cols, generator=g, device=DEV)
    return (v * scale).to(t)


def _product(a, b):
    """a b^T in 64 bits, and the root of the sum of squares of its terms"""
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=DEV)
    squares = torch.zeros_like(out)
    step = 1 << 17
    for k in range(0, a.shape[1], step):
        p, q = a[:, k:k + step].double(), b[:, k:k + step].double()
        out += p @ q.T
        squares += (p * p) @ (q * q).T
    return out, squares.sqrt()


def _check(got, a, b, one_sign, t):
    """got = a b^T, a and b with K along their rows"""
    want, rms = _product(a, b)
    K, half = a.shape[1], torch.finfo(t).eps / 2
    got = got.double()
    size = want.abs() if one_sign else 5 * rms
    off = (got - want).abs()
    assert (off <= _bound(K) * size + half * want.abs() + 2.0 ** -25).all(), (off / size).max().item()
    # the systematic part: the factor by which all results are too small
    factor = ((got * want).sum() / (want * want).sum()).item() - 1
    assert abs(factor) <= _bound(K) + 6 * half / math.sqrt(3 * want.numel()), factor


@pytest.mark.parametrize("one_sign", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, K, n_out", [(70, 1 << 21, 64), (33, (1 << 21) + 40, 130), (1200, 1 << 18, 1300), (2304, 70001, 2500), (300, 9000, 80),
                                            (2304, 8250, 2500), (2304, 12288, 2500)])
def test_forward(rows, K, n_out, dtype, one_sign):
    """Few rows with k split over a cluster, one tile a CTA, tiles of every width; also a K with an odd end."""
    t = TYPES[dtype]
    g = torch.Generator(device=DEV); g.manual_seed(rows + K)
    x, w = _operand(g, rows, K, 1.0, one_sign, t), _operand(g, n_out, K, 20.0 / K if one_sign else 1 / math.sqrt(K), one_sign, t)
    y = torch.full((rows, n_out), float("nan"), dtype=t, device=DEV)
    size = (rows, K, n_out, K, n_out)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size, t), dtype=torch.uint8, device=DEV)
    hpf.linear_fwd(x, w, None, None, y, None, *size, hpf.ACT_NONE, scratch)
    torch.cuda.synchronize()
    assert not hpf.linear_status(scratch)
    _check(y, x, w, one_sign, t)


@pytest.mark.parametrize("one_sign", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n_in, n_out", [(1 << 20, 72, 40), (150000, 1300, 264), (40, 136, 1 << 20), (520, 264, 300000)])
def test_gradients(rows, n_in, n_out, dtype, one_sign):
    """dW sums over the rows, dx over the outputs."""
    t = TYPES[dtype]
    g = torch.Generator(device=DEV); g.manual_seed(rows + n_out)
    K = max(rows, n_out)
    x, w = _operand(g, rows, n_in, 1.0, one_sign, t), _operand(g, n_out, n_in, 1.0, one_sign, t)
    dy = _operand(g, rows, n_out, 20.0 / K if one_sign else 1 / math.sqrt(K), one_sign, t)
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    size = (rows, n_in, n_out, n_in, n_out)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size, t), dtype=torch.uint8, device=DEV)
    hpf.linear_bwd(dy, None, x, w, dx, dw, None, *size, hpf.ACT_NONE, scratch)
    torch.cuda.synchronize()
    assert not hpf.linear_status(scratch)
    if rows > n_out:
        _check(dw, dy.T, x.T, one_sign, t)
    else:
        _check(dx, dy, w.T, one_sign, t)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, K, n_out, ld_y", [(9, 140000, 72, 72), (200, 20000, 1300, 1303), (1300, 8300, 4100, 4104), (2000, 9000, 2500, 2501)])
def test_write_out(rows, K, n_out, ld_y, dtype):
    """Bias, activation, kept z and residual behind a long sum; what lies between rows stays."""
    t = TYPES[dtype]
    g = torch.Generator(device=DEV); g.manual_seed(rows)
    x, w = _operand(g, rows, K, 1.0, False, t), _operand(g, n_out, K, 1 / math.sqrt(K), False, t)
    bias = _operand(g, 1, n_out, 0.3, False, t)[0].contiguous()
    y, z, r = (torch.full((rows, ld_y), 9.0, dtype=t, device=DEV) for _ in range(3))
    r[:, :n_out] = _operand(g, rows, n_out, 1.0, False, t)
    size = (rows, K, n_out, K, ld_y)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size, t), dtype=torch.uint8, device=DEV)
    hpf.linear_fwd(x, w, bias, r, y, z, *size, hpf.ACT_SILU, scratch)
    torch.cuda.synchronize()
    assert not hpf.linear_status(scratch)
    assert (y[:, n_out:] == 9.0).all() and (z[:, n_out:] == 9.0).all()
    want, rms = _product(x, w)
    want += bias.double()
    off = _bound(K) * 5 * rms + 2.0 ** -23 * (want.abs() + 1)
    half = torch.finfo(t).eps / 2
    assert ((z[:, :n_out].double() - want).abs() <= off + half * want.abs() + 2.0 ** -25).all()
    value = want * torch.sigmoid(want) + r[:, :n_out].double()
    assert ((y[:, :n_out].double() - value).abs() <= 1.2 * off + 2.0 ** -21 * want.abs() + 2.0 ** -22 * (value.abs() + 2) + half * value.abs() + 2.0 ** -25).all()


@pytest.mark.parametrize("rows, K, n_out", [(40, 300000, 64), (2304, 9000, 2500)])
def test_the_same_bits_again(rows, K, n_out):
    t = torch.bfloat16
    g = torch.Generator(device=DEV); g.manual_seed(rows)
    x, w = _operand(g, rows, K, 1.0, False, t), _operand(g, n_out, K, 1.0, False, t)
    ys = [torch.empty((rows, n_out), dtype=t, device=DEV) for _ in range(3)]
    size = (rows, K, n_out, K, n_out)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size, t), dtype=torch.uint8, device=DEV)
    for y in ys:
        hpf.linear_fwd(x, w, None, None, y, None, *size, hpf.ACT_NONE, scratch)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
