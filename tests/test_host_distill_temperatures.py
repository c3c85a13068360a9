"""Temperatures at which the loss of a distillation has no accuracy left, or T^2 no value, are refused before any CUDA call."""
import ctypes as C

import pytest

import paper_1911_05146_b200 as hpf

INVALID = -1
P = 1 << 12                     # an address that no refused call touches


def _statuses(t, rows):
    L = hpf.lib()
    t = C.c_float(t)
    return [L.hpf_distill_fwd(P, P, P, P, P, P, rows, 10, 10, 4, t, 0.5, 0, None),
            L.hpf_distill_bwd(P, P, P, P, P, P, 2 * P, rows, 10, 10, 10, 4, t, 0.5, 0, None),
            L.hpf_distill_fwd_bwd(P, P, P, P, P, P, 2 * P, rows, 10, 10, 10, 4, t, 0.5, 0, None)]


@pytest.mark.parametrize("t", [1e-30, 1e-6, 9.99e-4, 100.01, 1000.0, 1e20, 1e30, float("inf"), float("nan"), 0.0, -1.0])
def test_refused(t):
    assert _statuses(t, 4) == [INVALID] * 3
    assert b"0.001" in hpf.lib().hpf_last_error()


@pytest.mark.parametrize("t", [1e-3, 0.5, 1.0, 100.0])
def test_both_ends_are_accepted(t):
    assert _statuses(t, 0) == [0] * 3


def test_log_probabilities_keep_their_range():
    assert hpf.lib().hpf_logprobs_fwd(P, P, P, P, P, P, P, 0, 10, 10, 2, 1e30, 0, None) == 0
