"""A listed class whose logit is the type's lowest value: the loss is as large as the formula has it, where fp32 can hold that, at any temperature.

Bound: T (ln q - ln p) of such a class is its distance from the largest logit, exact but for fp32's step (2^-24), times q, which is off by 2^-20 + 4 2^-24 |t| / T (see
test_gpu_distill_temperatures), and alpha T; the other classes' parts are far smaller than the steps of that.
"""
import numpy as np
import pytest
import torch

import logits_reference as ref
import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T", [0.001, 0.5, 1.0, 2.5, 100.0])
@pytest.mark.parametrize("rows, n", [(4, 30), (4, 900), (4, 5000), (700, 2001)])
def test_the_loss_of_a_listed_class_at_the_lowest_value(rows, n, T, dtype):
    rng = np.random.Generator(np.random.PCG64(n))
    x = torch.from_numpy(rng.standard_normal((rows, n))).to(DEV).to(TYPES[dtype])
    x[:, 5] = torch.finfo(TYPES[dtype]).min
    k = 3
    ids = np.tile(np.array([[6, 5, 9]], np.int32), (rows, 1))
    t = np.tile(np.array([[1.0, 1.0, 0.5]], np.float32), (rows, 1))
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    w, loss, loss2, d = torch.ones(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(x)
    hpf.distill_fwd(x, None, dev(ids), dev(t), loss, None, rows, n, n, k, T, 1.0)
    hpf.distill_fwd_bwd(x, None, dev(ids), dev(t), w, loss2, d, rows, n, n, n, k, T, 1.0)
    torch.cuda.synchronize()
    T = float(np.float32(T))
    want, grad = ref.distill(x.double().cpu().numpy(), None, ids, t.astype(np.float64), np.ones(rows), T, 1.0)
    got = loss.double().cpu().numpy()
    assert torch.equal(loss, loss2)
    there = np.abs(want) < 3.4e38
    assert there.all() or T > 1
    assert np.all(np.isinf(got[~there])) and np.all(np.abs(got - want)[there] <= (2.0 ** -20 + 8 * 2.0 ** -24 / T + 2.0 ** -22) * np.abs(want)[there])
    assert torch.isfinite(d).all()
