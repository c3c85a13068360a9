"""Log-probabilities and distillation from their formulas in numpy, 64 bits, one row at a time (test infrastructure only)."""
import numpy as np

NINF = -np.inf


def distribution(s):
    """(p, ln p, lse) of one row of scaled logits; None without a finite one."""
    m = s.max()
    if m == NINF:
        return None
    e = np.exp(s - m)
    ln_sum = np.log(e.sum())        # kept apart from m: a row of the type's lowest value would swallow it
    return e / e.sum(), (s - m) - ln_sum, m + ln_sum


def logprobs(logits, labels, k, temperature):
    rows, n = logits.shape
    out = {"logprob": np.zeros(rows), "entropy": np.zeros(rows), "lse": np.full(rows, NINF), "ids": np.full((rows, k), -1), "top": np.full((rows, k), NINF)}
    for r in range(rows):
        d = distribution(logits[r] / temperature)
        there = 0 <= labels[r] < n
        if d is None:
            out["logprob"][r] = NINF if there else 0.0
            continue
        p, lp, out["lse"][r] = d
        out["entropy"][r] = -sum(a * b for a, b in zip(p[p > 0], lp[p > 0]))
        if there:
            out["logprob"][r] = lp[labels[r]]
        order = [c for c in sorted(range(n), key=lambda c: (-logits[r, c], c))[:k] if logits[r, c] > NINF]
        out["ids"][r, :len(order)], out["top"][r, :len(order)] = order, lp[order]
    return out


def logprobs_grad(logits, labels, d_logprob, d_entropy, temperature):
    out = np.zeros_like(logits)
    for r, row in enumerate(logits):
        d = distribution(row / temperature)
        there = 0 <= labels[r] < len(row)
        g, e = d_logprob[r] if there else 0.0, d_entropy[r]
        if d is None or (g == 0 and e == 0):
            continue
        p, lp, _ = d
        lp = np.where(p > 0, lp, 0.0)
        out[r] = -p * (g + e * (lp - (p * lp).sum()))
        if there:
            out[r, labels[r]] += g
    return out / temperature


def distill(logits, labels, ids, teacher, weight, temperature, alpha):
    """(loss, gradient) by row."""
    rows, n = logits.shape
    loss, grad = np.zeros(rows), np.zeros_like(logits)
    for r in range(rows):
        soft, hard = distribution(logits[r] / temperature), distribution(logits[r])
        if soft is None:
            continue
        there = (ids[r] >= 0) & (ids[r] < n)
        q = distribution(np.where(there, teacher[r] / temperature, NINF)) if len(ids[r]) else None
        if q is not None and alpha > 0:
            for j in np.nonzero(q[0] > 0)[0]:
                loss[r] += alpha * temperature ** 2 * q[0][j] * (q[1][j] - soft[1][ids[r][j]])
                grad[r, ids[r][j]] -= alpha * temperature * q[0][j]
            grad[r] += alpha * temperature * soft[0]
        if alpha < 1 and 0 <= labels[r] < n:
            loss[r] -= (1 - alpha) * hard[1][labels[r]]
            grad[r] += (1 - alpha) * hard[0]
            grad[r, labels[r]] -= 1 - alpha
        grad[r] *= weight[r]
    return loss, grad
