"""Distillation at the ends of its temperatures, 0.001 and 100, where T^2 is far from 1.

Bound.  loss = alpha T^2 sum_j q_j (ln q_j - ln p_j).  With |v| <= 4 the logits v / T lie within 4 / T: a logarithm is a difference (v - m) / T, rounded three times (and 1 / T
once more, 2^-24 relative each) less ln S, whose S is off by the exponentials' 2^-22 and a few 2^-24 a sum, at most 2^-20 in all:  2 (2^-20 + 4 * 2^-24 * 8 / T) a class for the two logarithms, and
q is off by 2^-20 + 4 * 2^-24 * 8 / T of itself.  A loss is off by alpha T^2 times that (plus that share of the sum of |q (ln q - ln p)|).  The gradient alpha T (p - q) is off by alpha T max(p, q)
times the same, rounded to the type.  The label's part, at temperature 1, is off by 1e-5.
"""
import numpy as np
import pytest
import torch

import logits_reference as ref
import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("alpha", [1.0, 0.5])
@pytest.mark.parametrize("T", [0.001, 0.01, 30.0, 100.0])
@pytest.mark.parametrize("rows, n", [(5, 2), (6, 10), (5, 256)])
def test_a_list_of_all_classes(rows, n, T, alpha):
    """The loss of a list that covers every class tends to a finite value as T grows (half the variance of the logits' differences)."""
    rng = np.random.Generator(np.random.PCG64(n))
    v = np.clip(rng.standard_normal((rows, n)), -4, 4).astype(np.float32)
    t = np.clip(rng.standard_normal((rows, n)), -4, 4).astype(np.float32)
    ids = np.stack([rng.permutation(n) for _ in range(rows)]).astype(np.int32)
    lab = rng.integers(0, n, rows).astype(np.int32)
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    x, w = dev(v), torch.ones(rows, device=DEV)
    loss, stats, loss2 = torch.empty(rows, device=DEV), torch.empty((rows, 2), device=DEV), torch.empty(rows, device=DEV)
    d, d2 = torch.empty_like(x), torch.empty_like(x)
    args = (x, dev(lab) if alpha < 1 else None, dev(ids), dev(t))
    hpf.distill_fwd(*args, loss, stats, rows, n, n, n, T, alpha)
    hpf.distill_bwd(*args, stats, w, d, rows, n, n, n, n, T, alpha)
    hpf.distill_fwd_bwd(*args, w, loss2, d2, rows, n, n, n, n, T, alpha)
    torch.cuda.synchronize()
    T = float(np.float32(T))
    loss_w, grad_w = ref.distill(v.astype(np.float64), lab, ids, t.astype(np.float64), np.ones(rows), T, alpha)
    one = 2.0 ** -20 + 4 * 2.0 ** -24 * 8 / T
    off = np.abs(loss.double().cpu().numpy() - loss_w)
    assert np.all(off <= alpha * T * T * 2 * one + one * np.abs(loss_w) + (1e-5 if alpha < 1 else 0)), off
    assert torch.equal(loss, loss2)
    for r in range(rows):
        q, p = ref.distribution(t[r].astype(np.float64) / T)[0], ref.distribution(v[r].astype(np.float64) / T)[0]
        most = p.copy()
        most[ids[r]] = np.maximum(most[ids[r]], q)
        for got in (d, d2):
            off = np.abs(got[r].double().cpu().numpy() - grad_w[r])
            # (a saved log-sum-exp below 128 adds 128 * 2^-24 to p)
            assert np.all(off <= alpha * T * most * (one + 2.0 ** -17) + (1e-5 if alpha < 1 else 0) + 2.0 ** -23 * np.abs(grad_w[r]) + 1e-12)
