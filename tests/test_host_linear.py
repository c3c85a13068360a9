"""Refusals and workspace sizes of the linear layer: decided before any CUDA call, so these run without a GPU."""
import ctypes as C

import pytest
import torch

import paper_1911_05146_b200 as hpf

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -4
P = 1 << 12                     # an address that no refused call touches


def _fwd(**kw):
    a = dict(x=P, w=P, bias=P, residual=P, y=P, z=P, rows=4, n_in=16, n_out=24, ld_x=16, ld_y=24, dtype=0, act=0, scratch=P, bytes=1 << 30)
    a.update(kw)
    return hpf.lib().hpf_linear_fwd(a["x"], a["w"], a["bias"], a["residual"], a["y"], a["z"], a["rows"], a["n_in"], a["n_out"], a["ld_x"], a["ld_y"],
                                    a["dtype"], a["act"], a["scratch"], a["bytes"], None)


def _bwd(**kw):
    a = dict(dy=P, z=P, x=P, w=P, dx=P, dw=P, db=P, rows=4, n_in=16, n_out=24, ld_x=16, ld_y=24, dtype=0, act=1, grad=0, scratch=P, bytes=1 << 30)
    a.update(kw)
    return hpf.lib().hpf_linear_bwd(a["dy"], a["z"], a["x"], a["w"], a["dx"], a["dw"], a["db"], a["rows"], a["n_in"], a["n_out"], a["ld_x"], a["ld_y"],
                                    a["dtype"], a["act"], a["grad"], a["scratch"], a["bytes"], None)


SIZES = [(dict(rows=-1), INVALID), (dict(n_in=0), INVALID), (dict(n_out=0), INVALID), (dict(ld_x=15), INVALID), (dict(ld_y=23), INVALID),
         (dict(dtype=3, grad=3), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(ld_x=1 << 40), UNSUPPORTED),
         (dict(rows=1 << 30, n_out=1 << 24, ld_y=1 << 24), UNSUPPORTED)]


@pytest.mark.parametrize("change, status", SIZES + [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(scratch=None), INVALID), (dict(x=P + 2), INVALID),
    (dict(w=P + 1, dtype=1), INVALID), (dict(bias=P + 2), INVALID), (dict(residual=P + 1), INVALID), (dict(bytes=255), WORKSPACE), (dict(scratch=P + 8), WORKSPACE),
    (dict(ld_x=17, bytes=300), WORKSPACE)])
def test_forward_refuses(change, status):
    change = {k: v for k, v in change.items() if k != "grad"}
    assert _fwd(**change) == status
    assert hpf.lib().hpf_last_error()


@pytest.mark.parametrize("change, status", SIZES + [
    (dict(dy=None), INVALID), (dict(z=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(scratch=None), INVALID), (dict(grad=1), INVALID),
    (dict(dtype=1, grad=2), INVALID), (dict(dw=P + 2), INVALID), (dict(dx=P + 2), INVALID), (dict(bytes=256), WORKSPACE)])
def test_backward_refuses(change, status):
    assert _bwd(**change) == status


def test_an_empty_batch_writes_nothing_forward():
    assert _fwd(rows=0, x=None, w=None, y=None, scratch=None) == 0
    assert _bwd(rows=0, dw=None, db=None) == 0


@pytest.mark.parametrize("dtype, e", [(torch.float32, 4), (torch.bfloat16, 2), (torch.float16, 2)])
def test_scratch_holds_dz_and_what_a_copy_cannot_address(dtype, e):
    up = lambda v: (v + 255) // 256 * 256  # noqa: E731
    pad = lambda n: (n * e + 127) // 128 * 128  # noqa: E731
    rows, n_in, n_out = 100, 64, 48
    assert hpf.linear_scratch_bytes(rows, n_in, n_out, n_in, n_out, dtype) == 256
    assert hpf.linear_scratch_bytes(rows, n_in, n_out, n_in, n_out, dtype, hpf.ACT_GELU) == 256 + up(rows * pad(n_out))
    assert hpf.linear_scratch_bytes(rows, n_in, n_out, n_in + 1, n_out, dtype) == 256 + up(rows * pad(n_in))
    odd = 256 + up(rows * pad(51)) + up(rows * pad(33)) + up(51 * pad(33))
    assert hpf.linear_scratch_bytes(rows, 33, 51, 33, 51, dtype) == odd
    assert hpf.linear_scratch_bytes(rows, 32, 48, 32, 48, dtype, aligned=False) == 256 + up(rows * pad(48)) + up(rows * pad(32)) + up(48 * pad(32))
    with pytest.raises(hpf.HpfError):
        hpf.linear_scratch_bytes(rows, 33, 51, 32, 51, dtype)
    with pytest.raises(hpf.HpfError):
        hpf.linear_scratch_bytes(rows, 33, 51, 33, 51, torch.float64)
    assert hpf.lib().hpf_linear_scratch_bytes(1, 1, 1, 1, 1, 0, 0, 1, C.POINTER(C.c_size_t)()) == INVALID


@pytest.mark.parametrize("change", [dict(y="x"), dict(y="w"), dict(y="bias"), dict(z="x"), dict(z="w"), dict(z="bias"), dict(z="residual"), dict(z="y")])
def test_forward_refuses_an_output_in_an_inputs_place(change):
    at = {name: P * (i + 1) for i, name in enumerate(["x", "w", "bias", "residual", "y", "z", "scratch"])}
    at.update({name: at[other] for name, other in change.items()})
    assert _fwd(**at) == INVALID


@pytest.mark.parametrize("change", [{o: i} for o in ("dx", "dw", "db") for i in ("dy", "z", "x", "w")] + [dict(dx="dw"), dict(dx="db"), dict(dw="db")])
def test_backward_refuses_an_output_in_an_inputs_place(change):
    at = {name: P * (i + 1) for i, name in enumerate(["dy", "z", "x", "w", "dx", "dw", "db", "scratch"])}
    at.update({name: at[other] for name, other in change.items()})
    assert _bwd(**at) == INVALID
