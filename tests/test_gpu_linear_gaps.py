"""Rows that start on 16-byte boundaries but do not end on them: what lies between rows is neither read nor written.

The tolerance is that of test_gpu_linear, whose cases are used: inputs and outputs are views of buffers that hold NaN between their rows.
"""
import pytest
import torch

import paper_1911_05146_b200 as hpf
from test_gpu_linear import TYPES, Case

pytestmark = pytest.mark.gpu


def _between(v, n, ld):
    return v.as_strided((v.shape[0] - 1, ld - n), (ld, 1), v.storage_offset() + n)


def _gap(n, unit):
    """columns to the next boundary and a boundary more for every other size"""
    return -n % unit + (unit if n % 3 == 0 else 0)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act, residual", [(hpf.ACT_NONE, False), (hpf.ACT_GELU, True)])
@pytest.mark.parametrize("rows, n_in, n_out", [(1, 41, 53), (3, 70, 1001), (40, 130, 67), (70, 77, 135), (200, 260, 197), (129, 1030, 257), (700, 301, 300), (1300, 517, 4100), (2500, 139, 4103)])
def test_rows_that_end_off_16_bytes(rows, n_in, n_out, act, residual, dtype):
    unit = 4 if dtype == "fp32" else 8
    gap_x, gap_y = _gap(n_in, unit), _gap(n_out, unit)
    c = Case(rows, n_in, n_out, dtype, act, gap_x=gap_x, gap_y=gap_y, residual=residual)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    if rows > 1:
        for v, n, gap in ((c.y, n_out, gap_y), (c.z_out, n_out, gap_y), (c.dx, n_in, gap_x)):
            if gap:
                assert torch.isnan(_between(v, n, n + gap)).all()
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n_in, n_out", [(5, 70, 53), (130, 70, 131), (2500, 139, 4103)])
def test_what_lies_behind_the_last_row_stays(rows, n_in, n_out, dtype):
    """y, z and dx end with their last column; other data follow at once."""
    unit = 4 if dtype == "fp32" else 8
    c = Case(rows, n_in, n_out, dtype, hpf.ACT_SILU, gap_x=-n_in % unit, gap_y=-n_out % unit, residual=False)
    ld_x, ld_y = c.size[3], c.size[4]
    bufs = [torch.full((rows * ld + 64,), 5.0, dtype=c.t, device="cuda:0") for ld in (ld_y, ld_y, ld_x)]
    y, z, dx = (b.as_strided((rows, n), (ld, 1)) for b, n, ld in zip(bufs, (n_out, n_out, n_in), (ld_y, ld_y, ld_x)))
    hpf.linear_fwd(c.x, c.w, c.bias, None, y, z, *c.size, c.act, c.scratch)
    hpf.linear_bwd(c.dy, c.z, c.x, c.w, dx, None, None, *c.size, c.act, c.scratch)
    c.forward(); c.backward()
    torch.cuda.synchronize()
    for b, v, n, ld, other in zip(bufs, (y, z, dx), (n_out, n_out, n_in), (ld_y, ld_y, ld_x), (c.y, c.z_out, c.dx)):
        assert torch.equal(v, other)
        assert (b[(rows - 1) * ld + n:] == 5.0).all()
        assert ld == n or (_between(v, n, ld) == 5.0).all()
