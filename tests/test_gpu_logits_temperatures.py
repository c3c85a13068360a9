"""Gradients of log-probability and entropy at the ends of the temperatures, where 1 / T^2 leaves fp32.

Bound.  d = -p (g + e (ln p + H)) / T (+ g / T at the label): p, ln p and H are each within 1e-5 of themselves (or absolutely, if they are below 1; see
test_gpu_logits), so d is within 3e-5 p (|g| + |e| (|ln p| + H + 1)) / T, and half a step of the type; where p is a label's, g's part besides.  What fp32 or the type has
only below its normal values may be lost: 2^-126 of p, and of d.
"""
import numpy as np
import pytest
import torch

import logits_reference as ref
import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("g, e", [(0.0, 1.0), (1.0, 0.0), (-0.7, 1.3)])
@pytest.mark.parametrize("T", [1e-30, 1e-20, 1e-10, 1e-3, 1.0, 1e5, 1e10, 1e19, 1e20, 1e30])
@pytest.mark.parametrize("rows, n", [(3, 1), (5, 20), (5, 900), (4, 3001), (200, 1500)])
def test_gradients_at_any_temperature(rows, n, T, g, e, dtype):
    rng = np.random.Generator(np.random.PCG64(n))
    x = torch.from_numpy(2.0 * rng.standard_normal((rows, n))).to(DEV).to(TYPES[dtype])
    if n > 10:
        x[0, 1::2] = float("-inf")
        x[1, :] = 0.5                                        # every class alike
        x[2, 3:] = torch.finfo(TYPES[dtype]).min
    v = x.double().cpu().numpy()
    lab = rng.integers(0, n, rows).astype(np.int32)
    lab[:3] = 0
    labels = torch.from_numpy(lab).to(DEV)
    full = lambda a: torch.full((rows,), a, device=DEV)  # noqa: E731
    lse, h, d = full(0.0), full(0.0), torch.full_like(x, 9.0)
    hpf.logprobs_fwd(x, labels, None, h, lse, None, None, rows, n, n, 0, T)
    hpf.logprobs_bwd(x, labels, lse, h, full(g) if g else None, full(e) if e else None, d, rows, n, n, n, T)
    torch.cuda.synchronize()
    T, g, e = (float(np.float32(a)) for a in (T, g, e))
    want = ref.logprobs_grad(v, lab, np.full(rows, g), np.full(rows, e), T)
    got, half = d.double().cpu().numpy(), torch.finfo(TYPES[dtype]).eps / 2
    assert np.isfinite(got).all()
    for r in range(rows):
        p, lp, _ = ref.distribution(v[r] / T)
        lp = np.where(p > 0, lp, 0.0)
        tol = (3e-5 * p + 2.0 ** -126) * (abs(g) + abs(e) * (np.abs(lp) + abs((p * lp).sum()) + 1)) / T + half * np.abs(want[r]) + 2.0 ** -126
        tol[lab[r]] += 3e-5 * abs(g) * p[lab[r]] / T
        assert np.all(np.abs(got[r] - want[r]) <= tol), (r, np.max(np.abs(got[r] - want[r]) / tol))


@pytest.mark.parametrize("T", [1e-30, 1e-10, 1e-5, 1.0, 1e5, 1e30])
@pytest.mark.parametrize("rows, n", [(5, 21), (5, 901), (4, 3001), (700, 1501)])
def test_masks_at_the_ends_of_rows_of_fp16(rows, n, T):
    """Rows of odd length start and end anywhere in a 16-byte unit; a gradient beyond 65504 is infinite, a masked class's is 0."""
    rng = np.random.Generator(np.random.PCG64(n))
    x = torch.from_numpy(2.0 * rng.standard_normal((rows, n))).to(DEV).half()
    x[:, :9] = float("-inf")
    x[:, n - 9:] = float("-inf")
    x[:, 11] = torch.finfo(torch.float16).min
    x[:, 12] = 10.0
    lab = np.full(rows, 12, np.int32)
    ones, lse, h, d = torch.ones(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.full_like(x, 9.0)
    hpf.logprobs_fwd(x, torch.from_numpy(lab).to(DEV), None, h, lse, None, None, rows, n, n, 0, T)
    hpf.logprobs_bwd(x, torch.from_numpy(lab).to(DEV), lse, h, ones, ones, d, rows, n, n, n, T)
    torch.cuda.synchronize()
    T = float(np.float32(T))
    v, got = x.double().cpu().numpy(), d.double().cpu().numpy()
    assert not np.isnan(got).any()
    assert np.all(got[np.isinf(v)] == 0)
    want = ref.logprobs_grad(v, lab, np.ones(rows), np.ones(rows), T)
    for r in range(0, rows, 50):
        p, lp, _ = ref.distribution(v[r] / T)
        lp = np.where(p > 0, lp, 0.0)
        tol = (3e-5 * p + 2.0 ** -126) * (2 + np.abs(lp) + abs((p * lp).sum())) / T + 2.0 ** -11 * np.abs(want[r]) + 2.0 ** -25
        tol[12] += 3e-5 * p[12] / T
        near = np.abs(want[r]) < 65000
        assert np.all(np.abs(got[r] - want[r])[near] <= tol[near])
        assert np.all(np.isinf(got[r][np.abs(want[r]) > 66000]))
