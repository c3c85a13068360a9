"""The bias gradient over very many rows: a sum of equal values must not drift.

Bound.  256 threads share the rows of a column (32 of a CTA, 8 CTAs).  Each adds up its rows one by one, up to 512, or, of more, blocks of 64 and then those, every addition
rounded to nearest: 2^-24 of the sum so far.  Their sums are joined in at most 16 additions.
"""
import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bound(rows):
    in_a_row = -(-rows // 256)
    return ((in_a_row if in_a_row <= 512 else 64 + in_a_row / 64 + 1) + 16) * 2.0 ** -24


@pytest.mark.parametrize("act", [hpf.ACT_NONE, hpf.ACT_RELU])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, n_out, ld_y", [(1 << 20, 8, 8), ((1 << 20) + 17, 5, 7), (300001, 70, 72), (16384, 64, 64), (40000, 33, 33), (131072, 33, 40), (131073, 33, 40), (131073, 40, 40)])
def test_a_sum_of_equal_values(rows, n_out, ld_y, dtype, act):
    size = (rows, 4, n_out, 4, ld_y, act)
    dy = torch.full((rows, ld_y), float("nan"), dtype=dtype, device=DEV)
    dy[:, :n_out] = torch.linspace(0.1, 0.9, n_out, device=DEV)
    z = torch.ones_like(dy) if act else None
    db = torch.empty(n_out, device=DEV)
    scratch = torch.zeros(hpf.linear_scratch_bytes(rows, 4, n_out, 4, ld_y, dtype, act), dtype=torch.uint8, device=DEV)
    hpf.linear_bwd(dy, z, None, None, None, None, db, *size, scratch)
    torch.cuda.synchronize()
    want = dy[0, :n_out].double() * rows
    assert ((db.double() - want).abs() <= (_bound(rows) + 2.0 ** -24) * want).all(), ((db.double() - want).abs() / want).max()


def test_values_of_both_signs():
    rows, n_out = 700000, 24
    g = torch.Generator(device=DEV); g.manual_seed(1)
    dy = torch.randn(rows, n_out, generator=g, device=DEV)
    db = torch.empty(n_out, device=DEV)
    scratch = torch.zeros(256, dtype=torch.uint8, device=DEV)
    hpf.linear_bwd(dy, None, None, None, None, None, db, rows, 4, n_out, 4, n_out, hpf.ACT_NONE, scratch)
    torch.cuda.synchronize()
    assert ((db.double() - dy.double().sum(0)).abs() <= _bound(rows) * dy.double().abs().sum(0)).all()
