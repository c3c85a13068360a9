"""Log-probabilities and distillation on the GPU against their formulas in 64 bits.

Tolerances.  Statistics are fp32: a log-probability is (v - m) / T - ln S with |v - m| / T up to about 40 (two roundings of 2^-24
relative), a ln S of a sum with relative error below 2^-20 (a few hundred fp32 additions a thread and the exponential's 2^-22 per term):
40 * 2^-23 + 2^-19 < 1e-5 absolute.  A lse below 128 is rounded once more: 128 * 2^-24.  A gradient is a sum of products p * (...), each
within a relative 1e-5 of its largest term, rounded to the tensor's type: half a step, eps / 2, of the value, plus half the smallest
subnormal step of fp16 (2^-25); bf16 and fp32 have none in reach.
"""
import numpy as np
import pytest
import torch

import paper_1911_05146_b200 as hpf
import logits_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
STAT = 1e-5


def _logits(rows, n, dtype, ld, offset, seed, kind="network"):
    """(tensor [rows][ld] flat view starting `offset` elements into its buffer, 64-bit values [rows][n])"""
    rng = np.random.Generator(np.random.PCG64(seed))
    v = 2.0 * rng.standard_normal((rows, n))
    if kind == "network":
        for r in range(rows):
            v[r, rng.integers(0, n, 4)] += 6.0
    elif kind == "equal":
        v[:] = 0.5
    elif kind == "few_values":
        v = np.round(v)
    elif kind == "falling":
        v = np.broadcast_to(8.0 - 16.0 * np.arange(n) / n, (rows, n)).copy()
    buf = torch.full((offset + rows * ld,), 77.0, dtype=TYPES[dtype], device=DEV)
    view = buf[offset:].as_strided((rows, n), (ld, 1))
    view.copy_(torch.from_numpy(v))
    return view, view.double().cpu().numpy()


def _labels(rows, n, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    lab = rng.integers(0, n, rows).astype(np.int32)
    lab[::5] = -1
    lab[1::7] = n          # outside: no label
    return torch.from_numpy(lab).to(DEV), lab


def _forward(x, labels, rows, n, ld, k, temperature, stream=None):
    o = {key: torch.full((rows,), 7.0, device=DEV) for key in ("logprob", "entropy", "lse")}
    ids, top = torch.full((rows, max(k, 1)), 7, dtype=torch.int32, device=DEV), torch.full((rows, max(k, 1)), 7.0, device=DEV)
    hpf.logprobs_fwd(x, labels, o["logprob"], o["entropy"], o["lse"], ids if k else None, top if k else None, rows, n, ld, k, temperature, stream)
    torch.cuda.synchronize()
    return {**{key: v.double().cpu().numpy() for key, v in o.items()}, "ids": ids.cpu().numpy()[:, :k], "top": top.double().cpu().numpy()[:, :k]}, o


def _close(got, want, tol):
    got, want = np.asarray(got), np.asarray(want)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), (got[~fine], want[~fine])
    tol, off = np.broadcast_to(tol, got.shape)[fine], np.abs(got[fine] - want[fine])
    assert np.all(off <= tol), np.max(off / tol)


def _check_forward(got, want):
    for key in ("logprob", "entropy", "top"):
        _close(got[key], want[key], STAT)
    _close(got["lse"], want["lse"], STAT + 2.0 ** -24 * np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0))
    assert np.array_equal(got["ids"], want["ids"])


def _grad_tol(want, dtype, scale):
    """half a step of the type, and 1e-5 of the row's scale times the class's own share of it"""
    tol = np.abs(want) * (torch.finfo(TYPES[dtype]).eps / 2 + 2e-5) + 1e-6 * scale
    return tol + (2.0 ** -25 if dtype == "fp16" else 0.0)


# one row to many, a class to long rows; odd strides, rows off 16-byte boundaries
SHAPES = [(1, 1, 1, 0), (3, 2, 5, 1), (5, 10, 10, 0), (7, 33, 40, 3), (4, 257, 257, 1), (3, 1000, 1001, 0), (2, 1024, 1024, 5), (3, 1025, 1025, 0),
          (2, 4099, 4101, 3), (1, 20011, 20011, 1), (2, 50021, 50021, 0), (150, 1500, 1501, 1), (160, 8195, 8195, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n, ld, offset", SHAPES)
def test_logprobs_forward_and_backward(rows, n, ld, offset, dtype):
    k, T = min(64, 3 + n // 7), 0.7
    x, v = _logits(rows, n, dtype, ld, offset, 11 * n + rows)
    labels, lab = _labels(rows, n, n)
    got, o = _forward(x, labels, rows, n, ld, k, T)
    want = ref.logprobs(v, lab, k, T)
    _check_forward(got, want)
    rng = np.random.Generator(np.random.PCG64(5))
    g, e = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    g[0] = e[0] = 0.0
    ld_d = n + 3
    d = torch.full((rows, ld_d), 9.0, dtype=x.dtype, device=DEV)
    dg, de = torch.from_numpy(g).to(DEV), torch.from_numpy(e).to(DEV)
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], dg, de, d, rows, n, ld, ld_d, T)
    torch.cuda.synchronize()
    dw = ref.logprobs_grad(v, lab, g.astype(np.float64), e.astype(np.float64), T)
    scale = (np.abs(g) + 20 * np.abs(e))[:, None] / T
    _close(d[:, :n].double().cpu().numpy(), dw, _grad_tol(dw, dtype, scale))
    assert torch.all(d[:, n:] == 9.0) and torch.all(d[0, :n] == 0)          # what lies between rows, and a row without weight
    # in place: the same bits
    xin = x.clone(memory_format=torch.contiguous_format)
    same = torch.empty((rows, n), dtype=x.dtype, device=DEV)
    hpf.logprobs_bwd(xin, labels, o["lse"], o["entropy"], dg, de, same, rows, n, n, n, T)
    hpf.logprobs_bwd(xin, labels, o["lse"], o["entropy"], dg, de, xin, rows, n, n, n, T)
    torch.cuda.synchronize()
    assert torch.equal(xin, same) and torch.equal(same, d[:, :n])


@pytest.mark.parametrize("kind", ["equal", "few_values", "falling"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows, n, k", [(2, 700, 64), (200, 5000, 64), (1, 60000, 64), (200, 20000, 1), (160, 3000, 20)])
def test_lists_of_rows_with_ties_and_of_sorted_rows(rows, n, k, dtype, kind):
    """Long runs of equal logits (the lower class first), and rows whose largest classes all stand together."""
    x, v = _logits(rows, n, dtype, n, 0, 3, kind)
    labels, lab = _labels(rows, n, 1)
    got, _ = _forward(x, labels, rows, n, n, k, 1.0)
    some = slice(0, 4)
    order = np.argsort(-v[some], axis=1, kind="stable")[:, :k]
    assert np.array_equal(got["ids"][some], order)
    assert np.array_equal(got["ids"], np.argsort(-v, axis=1, kind="stable")[:, :k])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("k", [1, 16, 17, 20, 63, 64])
@pytest.mark.parametrize("rows, n", [(9, 20), (9, 51), (700, 51), (9, 250), (9, 1000), (9, 1500), (300, 2000), (700, 2000), (9, 60001), (600, 5001), (150, 70001)])
def test_lists_with_fewer_classes_than_places(rows, n, k, dtype):
    """Rows of few classes, and rows whose mask leaves fewer classes than the list has places, or just as many, spread out or side by side."""
    x, _ = _logits(rows, n, dtype, n, 0, n + k)
    v = x.double().cpu().numpy().copy()
    rng = np.random.Generator(np.random.PCG64(k))
    some = min(rows, 9)
    for r, left in enumerate([n, 0, 1, k - 1, k, k + 1, k - 1, k, 2 * k][:some]):
        left = min(left, n)
        there = rng.choice(n, left, replace=False) if r < 6 else n // 2 - left // 2 + np.arange(left)
        masked = np.ones(n, bool)
        masked[there] = False
        v[r, masked] = -np.inf
    x.copy_(torch.from_numpy(v))
    labels, lab = _labels(rows, n, 1)
    got, _ = _forward(x, labels, rows, n, n, k, 1.0)
    order = np.argsort(-v, axis=1, kind="stable")[:, :k]
    want = np.full((rows, k), -1)
    want[:, : order.shape[1]] = np.where(np.isfinite(np.take_along_axis(v, order, 1)), order, -1)
    assert np.array_equal(got["ids"], want)
    assert np.array_equal(np.isfinite(got["top"]), want >= 0) and not np.isnan(got["top"]).any()
    _close(got["top"][:some], ref.logprobs(v[:some], lab[:some], k, 1.0)["top"], STAT)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n", [(6, 40), (6, 900), (6, 3001), (200, 1100)])
def test_masked_and_broken_rows(rows, n, dtype):
    """Rows that a mask leaves empty or almost empty, the type's lowest value as a mask, +inf and NaN."""
    x, v = _logits(rows, n, dtype, n, 0, 21)
    low = float(torch.finfo(TYPES[dtype]).min)
    x[0] = float("-inf")
    x[1] = float("-inf"); x[1, n - 1] = 1.5
    x[2, : n - 3] = low
    x[3] = low
    x[4, 1] = float("inf")
    x[5, 2] = float("nan")
    v = x.double().cpu().numpy()
    lab = np.zeros(rows, np.int32); lab[1] = n - 1
    labels = torch.from_numpy(lab).to(DEV)
    T, k = 1.0, 7
    got, o = _forward(x, labels, rows, n, n, k, T)
    whole = [r for r in range(rows) if r not in (4, 5)]
    want = ref.logprobs(v[whole], lab[whole], k, T)
    _close(got["entropy"][whole], want["entropy"], STAT)
    assert np.array_equal(got["ids"][whole], want["ids"])
    near = [i for i, r in enumerate(whole) if r != 3]
    _close(got["lse"][whole][near], want["lse"][near], STAT)
    for key in ("logprob", "top"):
        fine = np.where(np.isfinite(want[key]), want[key], 0)
        _close(got[key][whole], want[key], STAT + np.abs(fine) * 2.0 ** -22)
    assert np.all(np.isnan([got[key][r] for key in ("logprob", "entropy", "lse") for r in (4, 5)]))
    assert got["ids"][0].tolist() == [-1] * k and got["ids"][1].tolist() == [n - 1] + [-1] * (k - 1)
    assert got["ids"][4][0] == 1 and 2 not in got["ids"][5]
    ones = torch.ones(rows, device=DEV)
    d = torch.full_like(x, 9.0)
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], ones, ones, d, rows, n, n, n, T)
    torch.cuda.synchronize()
    dn = d.double().cpu().numpy()
    dw = ref.logprobs_grad(v[whole], lab[whole], np.ones(len(whole)), np.ones(len(whole)), T)
    _close(dn[whole], dw, _grad_tol(dw, dtype, 20.0))
    assert np.all(dn[0] == 0) and np.all(np.isnan(dn[[4, 5]]))
    # a padded batch: rows that weigh nothing get zeros whatever they hold
    ones[4:] = 0
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], ones, None, d, rows, n, n, n, T)
    torch.cuda.synchronize()
    assert torch.all(d[4:] == 0)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T", [1.0, 0.01, 300.0, 5000.0, 1e20])
@pytest.mark.parametrize("rows, n", [(5, 200), (5, 3100), (600, 1300)])
def test_masks_weigh_nothing_at_any_temperature(rows, n, T, dtype):
    """-inf and the type's lowest value next to each other, alone and among ordinary logits; at 5000 the lowest fp16 value is no mask any more."""
    x, _ = _logits(rows, n, dtype, n, 0, 41)
    low = float(torch.finfo(TYPES[dtype]).min)
    x[0, ::2] = float("-inf")
    x[1] = float("-inf"); x[1, 3:50:4] = low
    x[2, 1::2] = low; x[2, ::4] = float("-inf")
    x[3, :] = low; x[3, n // 2:] = float("-inf")
    v = x.double().cpu().numpy()
    lab = np.full(rows, 3, np.int32)
    labels = torch.from_numpy(lab).to(DEV)
    got, o = _forward(x, labels, rows, n, n, 5, T)
    want = ref.logprobs(v, lab, 5, T)
    _close(got["entropy"], want["entropy"], STAT)
    assert np.array_equal(got["ids"], want["ids"])
    # -1e30 and below times 1 / T may leave fp32: both sides are compared as fp32 has them
    as32 = lambda a: np.where(np.abs(a) > 3.4028235e38, np.sign(a) * np.inf, a)  # noqa: E731
    with np.errstate(invalid="ignore"):
        for key in ("logprob", "top"):
            w = as32(want[key])
            fine = np.isfinite(w)
            _close(got[key], w, STAT + np.where(fine, np.abs(w), 0) * 2.0 ** -22)
    ones, d = torch.ones(rows, device=DEV), torch.full_like(x, 9.0)
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], ones, ones, d, rows, n, n, n, T)
    dw = ref.logprobs_grad(v, lab, np.ones(rows), np.ones(rows), T)
    _close(d.double().cpu().numpy(), dw, _grad_tol(dw, dtype, 20.0 / T))


@pytest.mark.parametrize("shift", [0.0, 100.0, -1000.0, 30000.0])
@pytest.mark.parametrize("rows, n", [(3, 300), (3, 2500), (200, 1500)])
def test_large_logits_lose_nothing(rows, n, shift):
    """A shift changes no probability.  The saved lse cannot carry it in fp32 at 30000 (step 2^-9): the backward pass must not need it to."""
    x, v = _logits(rows, n, "fp32", n, 0, 31)
    x += shift
    v = x.double().cpu().numpy()
    labels, lab = _labels(rows, n, 2)
    got, o = _forward(x, labels, rows, n, n, 5, 1.0)
    _check_forward(got, ref.logprobs(v, lab, 5, 1.0))
    ones, d = torch.ones(rows, device=DEV), torch.empty_like(x)
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], ones, ones, d, rows, n, n, n, 1.0)
    dw = ref.logprobs_grad(v, lab, np.ones(rows), np.ones(rows), 1.0)
    _close(d.double().cpu().numpy(), dw, _grad_tol(dw, "fp32", 20.0))


def _teacher(rows, n, k, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    ids = np.stack([rng.permutation(max(n, k))[:k] for _ in range(rows)]).astype(np.int32)
    ids[ids >= n] = -1
    t = (3.0 * rng.standard_normal((rows, k))).astype(np.float32)
    if k > 3:
        ids[0, 1] = ids[0, 0]          # the same class twice
        ids[-1, 2] = n + 5             # outside
        t[-1, 3] = -np.inf             # listed, but masked
    if rows > 2:
        ids[1] = -1                    # a list that holds nothing
    return torch.from_numpy(ids).to(DEV), torch.from_numpy(t).to(DEV), ids, t.astype(np.float64)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("alpha, T", [(1.0, 2.0), (0.3, 4.0), (0.0, 1.0)])
@pytest.mark.parametrize("rows, n, ld, offset, k", [(1, 1, 1, 0, 1), (4, 10, 10, 0, 4), (5, 300, 307, 3, 256), (3, 1000, 1000, 0, 16), (3, 2049, 2051, 1, 20),
                                                    (1, 30011, 30011, 0, 64), (150, 1201, 1201, 1, 8)])
def test_distill(rows, n, ld, offset, k, alpha, T, dtype):
    x, v = _logits(rows, n, dtype, ld, offset, 7 * n + k)
    labels, lab = _labels(rows, n, 3)
    ids, t, ids_h, t_h = _teacher(rows, n, k, 9)
    w = np.random.Generator(np.random.PCG64(4)).standard_normal(rows).astype(np.float32)
    if rows > 3:
        w[3] = 0.0
    loss_w, grad_w = ref.distill(v, lab, ids_h, t_h, w.astype(np.float64), T, alpha)
    weight = torch.from_numpy(w).to(DEV)
    loss, stats = torch.full((rows,), 7.0, device=DEV), torch.empty((rows, 2), device=DEV)
    lab_arg = labels if alpha < 1 else None
    hpf.distill_fwd(x, lab_arg, ids, t, loss, stats, rows, n, ld, k, T, alpha)
    # a loss is a sum of up to k products of q and differences of logarithms below 40, each within 1e-5, times alpha T^2
    tol = 3e-5 * max(1.0, T * T) + 1e-5 * np.abs(loss_w)
    _close(loss.double().cpu().numpy(), loss_w, tol)
    ld_d = ld + 1
    d = torch.full((rows, ld_d), 9.0, dtype=x.dtype, device=DEV)
    hpf.distill_bwd(x, lab_arg, ids, t, stats, weight, d, rows, n, ld, ld_d, k, T, alpha)
    gt = _grad_tol(grad_w, dtype, np.abs(w)[:, None] * max(1.0, T) * 3)
    _close(d[:, :n].double().cpu().numpy(), grad_w, gt)
    assert torch.all(d[:, n:] == 9.0)
    both, loss2 = torch.full((rows, ld_d), 9.0, dtype=x.dtype, device=DEV), torch.full((rows,), 7.0, device=DEV)
    hpf.distill_fwd_bwd(x, lab_arg, ids, t, weight, loss2, both, rows, n, ld, ld_d, k, T, alpha)
    _close(both[:, :n].double().cpu().numpy(), grad_w, gt)
    assert torch.equal(loss, loss2) and torch.all(both[:, n:] == 9.0)
    xin = x.clone(memory_format=torch.contiguous_format)
    same = torch.empty((rows, n), dtype=x.dtype, device=DEV)
    hpf.distill_fwd_bwd(xin, lab_arg, ids, t, weight, loss2, same, rows, n, n, n, k, T, alpha)
    hpf.distill_fwd_bwd(xin, lab_arg, ids, t, weight, loss2, xin, rows, n, n, n, k, T, alpha)     # in place
    torch.cuda.synchronize()
    assert torch.equal(xin, same)


@pytest.mark.parametrize("rows, n", [(6, 30), (6, 1025), (200, 1100)])
def test_distill_of_masked_rows(rows, n):
    x, _ = _logits(rows, n, "bf16", n, 0, 8)
    x[0] = float("-inf")
    x[1, 5] = float("-inf")
    x[2] = torch.finfo(torch.bfloat16).min
    x[3] = float("nan")
    v = x.double().cpu().numpy()
    k, T = 4, 2.0
    ids = np.tile(np.array([[5, 6, 7, 8]], np.int32), (rows, 1))
    t = np.zeros((rows, k), np.float32)
    lab = np.full(rows, 6, np.int32)
    w = np.ones(rows, np.float32); w[3] = 0
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    loss, stats, d, d2 = torch.empty(rows, device=DEV), torch.empty((rows, 2), device=DEV), torch.empty_like(x), torch.empty_like(x)
    args = (dev(lab), dev(ids), dev(t))
    hpf.distill_fwd_bwd(x, *args, dev(w), loss, d, rows, n, n, n, k, T, 0.5)
    hpf.distill_fwd(x, *args, loss, stats, rows, n, n, k, T, 0.5)
    hpf.distill_bwd(x, *args, stats, dev(w), d2, rows, n, n, n, k, T, 0.5)
    v[3] = 0.0
    loss_w, grad_w = ref.distill(v, lab, ids, t.astype(np.float64), w.astype(np.float64), T, 0.5)
    assert loss[0] == 0 and torch.isinf(loss[1]) and loss[1] > 0 and torch.isnan(loss[3])
    keep = [r for r in range(rows) if r != 3]
    _close(loss.double().cpu().numpy()[keep], loss_w[keep], 1e-4)
    for g in (d, d2):
        assert torch.all(g[0] == 0) and torch.all(g[3] == 0)
        _close(g.double().cpu().numpy(), grad_w, _grad_tol(grad_w, "bf16", 6.0))


def test_gradients_against_differences():
    """Central differences of the forward calls' own outputs (fp32, step 2^-5: the third derivative of each is below 2)."""
    rows, n, k, T, alpha, h = 2, 12, 3, 1.5, 0.6, 2.0 ** -5
    x, _ = _logits(rows, n, "fp32", n, 0, 77)
    lab = torch.tensor([3, 11], dtype=torch.int32, device=DEV)
    ids = torch.tensor([[0, 3, 7], [1, 2, 11]], dtype=torch.int32, device=DEV)
    t = torch.tensor([[1.0, 0.0, 2.0], [0.5, 0.5, -1.0]], device=DEV)
    one = torch.ones(rows, device=DEV)
    loss, d = torch.empty(rows, device=DEV), torch.empty_like(x)
    hpf.distill_fwd_bwd(x, lab, ids, t, one, loss, d, rows, n, n, n, k, T, alpha)
    _, o = _forward(x, lab, rows, n, n, 0, T)
    dl, dh = torch.empty_like(x), torch.empty_like(x)
    hpf.logprobs_bwd(x, lab, o["lse"], o["entropy"], one, None, dl, rows, n, n, n, T)
    hpf.logprobs_bwd(x, lab, o["lse"], o["entropy"], None, one, dh, rows, n, n, n, T)
    for c in range(n):
        ends = []
        for sign in (1, -1):
            y = x.clone(); y[:, c] += sign * h
            l1 = torch.empty(rows, device=DEV)
            hpf.distill_fwd(y, lab, ids, t, l1, None, rows, n, n, k, T, alpha)
            f, _ = _forward(y, lab, rows, n, n, 0, T)
            ends.append((l1.double().cpu().numpy(), f["logprob"], f["entropy"]))
        for got, a, b in zip((d, dl, dh), ends[0], ends[1]):
            # h^2 / 6 * 2 from the third derivative, 2 * 1e-5 / (2 h) from the two values' rounding
            assert np.all(np.abs(got[:, c].double().cpu().numpy() - (a - b) / (2 * h)) <= 2 * h * h / 6 + 2 * STAT / (2 * h))


def test_streams_graphs_and_repeats():
    """The same bits on another stream, in a replayed graph with new inputs, and twice in a row."""
    rows, n, k, T = 37, 5003, 12, 1.3
    x, v = _logits(rows, n, "bf16", n, 0, 1)
    labels, lab = _labels(rows, n, 1)
    ids, t, *_ = _teacher(rows, n, k, 2)
    w = torch.ones(rows, device=DEV)

    def call(bufs):
        hpf.logprobs_fwd(x, labels, bufs["lp"], bufs["h"], bufs["lse"], bufs["ids"], bufs["top"], rows, n, n, k, T)
        hpf.logprobs_bwd(x, labels, bufs["lse"], bufs["h"], w, w, bufs["d1"], rows, n, n, n, T)
        hpf.distill_fwd_bwd(x, labels, ids, t, w, bufs["loss"], bufs["d2"], rows, n, n, n, k, T, 0.5)

    def buffers():
        f = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
        return {"lp": f(rows), "h": f(rows), "lse": f(rows), "loss": f(rows), "top": f(rows, k), "ids": torch.zeros((rows, k), dtype=torch.int32, device=DEV),
                "d1": torch.zeros_like(x), "d2": torch.zeros_like(x)}

    eager, side, graphed = buffers(), buffers(), buffers()
    call(eager)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(side)
    torch.cuda.synchronize()
    assert all(torch.equal(eager[key], side[key]) for key in eager)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(graphed)
    for _ in range(2):
        x.copy_(x.flip(1).contiguous())
        g.replay()
        call(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(eager[key], graphed[key]) for key in eager)


def test_binding_refuses_what_the_kernels_would_misread():
    x = torch.zeros((2, 10), dtype=torch.float64, device=DEV)
    f = torch.zeros(2, device=DEV)
    with pytest.raises(hpf.HpfError):
        hpf.logprobs_fwd(x, None, None, f, None, None, None, 2, 10, 10)
    x = x.float()
    with pytest.raises(hpf.HpfError):
        hpf.logprobs_fwd(x, torch.zeros(2, dtype=torch.int64, device=DEV), f, None, None, None, None, 2, 10, 10)
    with pytest.raises(hpf.HpfError):
        hpf.logprobs_fwd(x.cpu(), None, None, f, None, None, None, 2, 10, 10)
    with pytest.raises(hpf.HpfError):
        hpf.distill_fwd_bwd(x, None, None, None, f, f, torch.zeros((2, 10), dtype=torch.bfloat16, device=DEV), 2, 10, 10, 10, 0, 1.0, 1.0)


def test_offsets_beyond_32_bits():
    """Rows that start more than 2^32 elements into the buffer."""
    n, ld, rows = 1030, (1 << 31) + 8, 3
    buf = torch.empty((rows - 1) * ld + n, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((rows, n), (ld, 1))
    v = np.random.Generator(np.random.PCG64(6)).standard_normal((rows, n))
    x.copy_(torch.from_numpy(v))
    v = x.double().cpu().numpy()
    lab = np.arange(rows, dtype=np.int32)
    labels = torch.from_numpy(lab).to(DEV)
    got, o = _forward(x, labels, rows, n, ld, 9, 1.0)
    _check_forward(got, ref.logprobs(v, lab, 9, 1.0))
    one = torch.ones(rows, device=DEV)
    hpf.logprobs_bwd(x, labels, o["lse"], o["entropy"], one, one, x, rows, n, ld, ld, 1.0)
    dw = ref.logprobs_grad(v, lab, np.ones(rows), np.ones(rows), 1.0)
    _close(x.double().cpu().numpy(), dw, _grad_tol(dw, "bf16", 20.0))


@pytest.mark.parametrize("alpha, T", [(1.0, 1.7), (0.4, 1.0), (0.4, 2.0), (0.4, 3.0), (0.4, 4.0), (0.4, 0.9)])
@pytest.mark.parametrize("rows, n, ld, offset, dtype, k", [(1200, 33001, 33001, 0, "bf16", 20), (910, 120007, 120011, 3, "fp16", 64), (900, 62003, 62003, 1, "fp32", 200),
                                                           (1000, 106496, 106496, 0, "bf16", 7), (893, 110001, 110003, 5, "bf16", 256)])
def test_distill_of_many_long_rows(rows, n, ld, offset, dtype, k, alpha, T):
    """Several waves of rows on either side of the lengths at which the CTAs change, from any alignment, with masked, broken and weightless rows among
    them.  Sampled rows against 64 bits, all of them against the two separate calls; in place the same bits."""
    t = TYPES[dtype]
    g = torch.Generator(device=DEV); g.manual_seed(n)
    buf = torch.full((offset + rows * ld,), 77.0, dtype=t, device=DEV)
    x = buf[offset:].as_strided((rows, n), (ld, 1))
    x.copy_(2.0 * torch.randn(rows, n, generator=g, device=DEV))
    x[1] = float("-inf")
    x[2, 5:] = float("-inf")
    x[3, 7] = float("nan")
    x[4] = torch.finfo(t).min
    x[rows - 1] += 300.0
    labels = torch.randint(n, (rows,), generator=g, device=DEV, dtype=torch.int32)
    labels[::5] = -1
    labels[2] = 3
    ids = torch.randint(n, (rows, k), generator=g, device=DEV, dtype=torch.int32)
    ids[2] = 1
    ids[7] = -1
    teacher = 3.0 * torch.randn(rows, k, generator=g, device=DEV)
    w = torch.randn(rows, generator=g, device=DEV)
    w[3] = 0.0
    w[8] = 0.0
    lab = labels if alpha < 1 else None
    loss, loss2, stats = torch.full((rows,), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV), torch.empty((rows, 2), device=DEV)
    ld_d = ld + 3
    d = torch.full((rows, ld_d), 9.0, dtype=t, device=DEV)
    d2 = torch.empty((rows, ld), dtype=t, device=DEV)
    hpf.distill_fwd_bwd(x, lab, ids, teacher, w, loss, d, rows, n, ld, ld_d, k, T, alpha)
    hpf.distill_fwd(x, lab, ids, teacher, loss2, stats, rows, n, ld, k, T, alpha)
    hpf.distill_bwd(x, lab, ids, teacher, stats, w, d2, rows, n, ld, ld, k, T, alpha)
    torch.cuda.synchronize()
    assert (d[:, n:] == 9.0).all()
    some = [0, 1, 2, 4, 5, 7, 8, 9, rows // 2, rows - 2, rows - 1]
    pick = torch.tensor(some, device=DEV)
    v = x[pick].double().cpu().numpy()
    h = lambda a: a[pick].cpu().numpy()  # noqa: E731
    loss_w, grad_w = ref.distill(v, h(labels), h(ids), h(teacher).astype(np.float64), h(w).astype(np.float64), T, alpha)
    _close(loss[pick].double().cpu().numpy(), loss_w, 3e-5 * max(1.0, T * T) + 1e-5 * np.abs(np.where(np.isfinite(loss_w), loss_w, 0)))
    gt = _grad_tol(grad_w, dtype, np.abs(h(w))[:, None] * max(1.0, T) * 3)
    _close(d[pick][:, :n].double().cpu().numpy(), grad_w, gt)
    # both ways are within their tolerance of the same value; rows of a few large probabilities apart, half a step of the type each
    ok = torch.isfinite(loss2)
    assert torch.equal(torch.isnan(loss), torch.isnan(loss2)) and torch.isnan(loss[3])
    assert ((loss - loss2).abs()[ok] <= 6e-5 * max(1.0, T * T) + 2e-5 * loss2.abs()[ok]).all()
    a, b = d[:, :n].float(), d2[:, :n].float()
    step = float(torch.finfo(t).eps) + 4e-5
    bound = step * torch.maximum(a.abs(), b.abs()) + 2e-6 * 3 * max(1.0, T) * w.abs()[:, None] + (2.0 ** -24 if dtype == "fp16" else 0.0)
    assert ((a - b).abs() <= bound).all()
    del a, b, bound, d2
    loss3 = torch.empty(rows, device=DEV)
    hpf.distill_fwd_bwd(x, lab, ids, teacher, w, loss3, x, rows, n, ld, ld, k, T, alpha)
    torch.cuda.synchronize()
    assert torch.equal(x, d[:, :n]) and torch.equal(loss3[ok], loss[ok])
    assert (buf[:offset] == 77.0).all() and (ld == n or (buf[offset:].as_strided((rows - 1, ld - n), (ld, 1), offset + n) == 77.0).all())
