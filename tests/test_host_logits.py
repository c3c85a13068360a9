"""Refusals of the log-probability and distillation entry points: they return before any CUDA call, so these run without a GPU."""
import pytest

import paper_1911_05146_b200 as hpf

INVALID, UNSUPPORTED = -1, -2
P = 1 << 12                     # an address that no refused call touches


def _fwd(**kw):
    a = dict(logits=P, labels=P, logprob=P, entropy=P, lse=P, ids=P, lps=P, rows=4, classes=10, ld=10, k=2, t=1.0, dtype=0)
    a.update(kw)
    return hpf.lib().hpf_logprobs_fwd(a["logits"], a["labels"], a["logprob"], a["entropy"], a["lse"], a["ids"], a["lps"], a["rows"], a["classes"],
                                      a["ld"], a["k"], a["t"], a["dtype"], None)


@pytest.mark.parametrize("change, status", [
    (dict(logits=None), INVALID), (dict(labels=None), INVALID), (dict(ids=None), INVALID), (dict(lps=None), INVALID), (dict(rows=-1), INVALID),
    (dict(classes=0), INVALID), (dict(ld=9), INVALID), (dict(k=-1), UNSUPPORTED), (dict(k=65), UNSUPPORTED), (dict(t=0.0), INVALID),
    (dict(t=-1.0), INVALID), (dict(t=float("nan")), INVALID), (dict(t=float("inf")), INVALID), (dict(t=1e-45), INVALID), (dict(t=1e31), INVALID), (dict(dtype=3), INVALID),
    (dict(logits=P + 2), INVALID), (dict(logits=P + 1, dtype=1), INVALID), (dict(rows=1 << 40), UNSUPPORTED)])
def test_logprobs_fwd_refuses(change, status):
    assert _fwd(**change) == status
    assert hpf.lib().hpf_last_error()


def test_no_rows_is_no_work():
    """An empty batch needs no device and no buffers."""
    assert _fwd(rows=0, logits=None) == 0
    assert hpf.lib().hpf_logprobs_bwd(None, None, None, None, None, None, None, 0, 10, 10, 10, 1.0, 0, None) == 0
    assert hpf.lib().hpf_distill_fwd(None, None, None, None, None, None, 0, 10, 10, 4, 1.0, 0.5, 0, None) == 0
    assert hpf.lib().hpf_distill_bwd(None, None, None, None, None, None, None, 0, 10, 10, 10, 4, 1.0, 0.5, 0, None) == 0
    assert hpf.lib().hpf_distill_fwd_bwd(None, None, None, None, None, None, None, 0, 10, 10, 10, 4, 1.0, 0.5, 0, None) == 0


@pytest.mark.parametrize("change, status", [
    (dict(logits=None), INVALID), (dict(lse=None), INVALID), (dict(out=None), INVALID), (dict(labels=None), INVALID), (dict(entropy=None), INVALID),
    (dict(ld_d=9), INVALID), (dict(out=P + 2), INVALID), (dict(t=0.0), INVALID), (dict(dtype=-1), INVALID)])
def test_logprobs_bwd_refuses(change, status):
    a = dict(logits=P, labels=P, lse=P, entropy=P, g=P, e=P, out=P, ld_d=10, t=1.0, dtype=0)
    a.update(change)
    assert hpf.lib().hpf_logprobs_bwd(a["logits"], a["labels"], a["lse"], a["entropy"], a["g"], a["e"], a["out"], 4, 10, 10, a["ld_d"], a["t"], a["dtype"], None) == status


@pytest.mark.parametrize("change, status", [
    (dict(logits=None), INVALID), (dict(labels=None), INVALID), (dict(ids=None), INVALID), (dict(teacher=None), INVALID), (dict(alpha=-0.1), INVALID),
    (dict(alpha=1.1), INVALID), (dict(alpha=float("nan")), INVALID), (dict(t=0.0), INVALID), (dict(k=257), UNSUPPORTED), (dict(k=-1), UNSUPPORTED),
    (dict(loss=None), INVALID), (dict(out=None), INVALID), (dict(w=None), INVALID), (dict(ld_d=9), INVALID), (dict(dtype=7), INVALID)])
def test_distill_refuses(change, status):
    a = dict(logits=P, labels=P, ids=P, teacher=P, w=P, loss=P, out=P, ld_d=10, k=4, t=1.0, alpha=0.5, dtype=0)
    a.update(change)
    L = hpf.lib()
    assert L.hpf_distill_fwd_bwd(a["logits"], a["labels"], a["ids"], a["teacher"], a["w"], a["loss"], a["out"], 4, 10, 10, a["ld_d"], a["k"], a["t"],
                                 a["alpha"], a["dtype"], None) == status
    if not {"w", "out", "ld_d"} & set(change):
        assert L.hpf_distill_fwd(a["logits"], a["labels"], a["ids"], a["teacher"], a["loss"], P, 4, 10, 10, a["k"], a["t"], a["alpha"], a["dtype"], None) == status
    if "loss" not in change:
        assert L.hpf_distill_bwd(a["logits"], a["labels"], a["ids"], a["teacher"], P, a["w"], a["out"], 4, 10, 10, a["ld_d"], a["k"], a["t"], a["alpha"],
                                 a["dtype"], None) == status


@pytest.mark.parametrize("name", ["labels", "logprob", "entropy", "lse", "ids", "lps"])
def test_logprobs_fwd_refuses_words_off_their_boundary(name):
    assert _fwd(**{name: P + 2}) == INVALID


def test_gradients_refuse_words_off_their_boundary_and_another_stride_in_place():
    L, other = hpf.lib(), 2 * P
    for i in range(1, 6):
        assert L.hpf_logprobs_bwd(*[P + 2 if j == i else P for j in range(6)], other, 4, 10, 10, 10, 1.0, 0, None) == INVALID
        assert L.hpf_distill_bwd(*[P + 2 if j == i else P for j in range(6)], other, 4, 10, 10, 10, 4, 1.0, 0.5, 0, None) == INVALID
        assert L.hpf_distill_fwd_bwd(*[P + 2 if j == i else P for j in range(6)], other, 4, 10, 10, 10, 4, 1.0, 0.5, 0, None) == INVALID
        assert L.hpf_distill_fwd(*[P + 2 if j == i else P for j in range(6)], 4, 10, 10, 4, 1.0, 0.5, 0, None) == INVALID
    assert L.hpf_logprobs_bwd(*[P] * 7, 4, 10, 10, 11, 1.0, 0, None) == INVALID
    assert L.hpf_distill_bwd(*[P] * 7, 4, 10, 10, 11, 4, 1.0, 0.5, 0, None) == INVALID
    assert L.hpf_distill_fwd_bwd(*[P] * 7, 4, 10, 12, 10, 4, 1.0, 0.5, 0, None) == INVALID
