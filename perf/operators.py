"""The linear layer, label log-probabilities and distillation as cases that can be timed.

A "linear" case is a matrix product with bias, activation and residual, forward alone or with its gradients.  A "logprobs"
case scores given labels (log-probability, entropy, the k likeliest classes), with the gradient where it says so.  A
"distill" case is the loss against a teacher's k largest logits mixed with cross-entropy on the labels, and its gradient.
With `own` false the operators are spelled out in torch in 32 bits; with `own` true they are the library's calls.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")


# ---- the cases -------------------------------------------------------------------------------------------------------
def _linear(name, rows, n_in, n_out, dtype, act, residual, train):
    return {"name": name, "op": "linear", "rows": rows, "in": n_in, "out": n_out, "type": dtype, "act": act, "residual": residual, "train": train}


def _logprobs(name, rows, classes, dtype, k, temperature, train):
    return {"name": name, "op": "logprobs", "rows": rows, "classes": classes, "type": dtype, "k": k, "temperature": temperature, "train": train}


def _distill(name, rows, classes, dtype, k, temperature, alpha, fused):
    return {"name": name, "op": "distill", "rows": rows, "classes": classes, "type": dtype, "k": k, "temperature": temperature, "alpha": alpha, "fused": fused}


def listed():
    return [
        # one sample served through a wide layer: the weights are read once and that is all there is
        _linear("linear_one_row_bf16", 1, 4096, 16384, "bf16", "gelu", False, False),
        # the head of a network for large images in training: 64 samples of a micro-batch, a thousand classes, fp32
        _linear("linear_head1000_b64_fp32", 64, 2048, 1000, "fp32", "none", False, True),
        # a large fully connected layer behind convolutions, trained: weights and their gradient outweigh the batch
        _linear("linear_fc4096_b128_bf16", 128, 4096, 4096, "bf16", "relu", False, True),
        # the output layer of a model with very many classes, nothing divides evenly
        _linear("linear_logits50021_fp16", 509, 1024, 50021, "fp16", "none", False, True),
        # a wide layer of a large model with a long batch: bound by the tensor cores
        _linear("linear_wide_8192_bf16", 8192, 4096, 16384, "bf16", "gelu", True, True),
        # the predictions on a batch of small images, with the five likeliest classes: the smallest call
        _logprobs("logprobs_10_b128_fp32", 128, 10, "fp32", 5, 1.0, False),
        # one new token of a large vocabulary, with its alternatives: latency
        _logprobs("logprobs_one_row_bf16", 1, 131071, "bf16", 20, 1.0, False),
        # scoring a corpus, or a teacher that writes down its list: rows of an odd length
        _logprobs("logprobs_score50021_bf16", 4096, 50021, "bf16", 8, 1.0, False),
        # training on log-probabilities and entropy at a sampling temperature, fp32 logits
        _logprobs("logprobs_train32000_fp32", 2048, 32000, "fp32", 0, 0.7, True),
        # distilling a classifier of a thousand classes
        _distill("distill_1000_b256_fp32", 256, 1000, "fp32", 16, 4.0, 0.7, True),
        # the same with the backward pass called later, rows of an odd length
        _distill("distill_32003_fp16", 777, 32003, "fp16", 20, 1.5, 1.0, False),
        # distilling a large vocabulary over a long batch: one pass over logits larger than any cache
        _distill("distill_128000_bf16", 4096, 128000, "bf16", 64, 2.0, 0.5, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(("fp32", "bf16", "bf16", "fp16"))
    op = rng.choice(("linear", "linear", "logprobs", "distill"))
    if op == "linear":
        while True:
            case = _linear("", _log(rng, 1, 16384), _log(rng, 16, 16384), _log(rng, 10, 65536), dtype, rng.choice(ACTS), rng.random() < 0.4, rng.random() < 0.7)
            for k in ("in", "out"):
                if rng.random() < 0.5 and case[k] >= 128:
                    case[k] = case[k] // 64 * 64
            w = work(case)
            if w["flops"] <= 1.5e12 and w["bytes"] <= 1.5e9:
                break
    else:
        while True:
            rows, classes = _log(rng, 1, 8192), _log(rng, 10, 131072)
            if rows * classes <= 300_000_000:
                break
        if op == "logprobs":
            case = _logprobs("", rows, classes, dtype, rng.choice((0, 1, 5, 8, 20, 64)), rng.choice((1.0, 1.0, 0.7, 1.3)), rng.random() < 0.5)
        else:
            case = _distill("", rows, classes, dtype, rng.choice((1, 8, 20, 64, 200)), rng.choice((1.0, 2.0, 3.0, 4.0)), rng.choice((1.0, 0.9, 0.5)), rng.random() < 0.7)
    case.pop("name")
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    dtype, rows = TYPES[case["type"]], case["rows"]
    s = {"case": case}
    if case["op"] == "linear":
        n_in, n_out = case["in"], case["out"]
        s["x"] = normal(rows, n_in).to(dtype)
        s["w"] = (normal(n_out, n_in) * math.sqrt(2.0 / n_in)).to(dtype)
        s["bias"] = (0.1 * normal(n_out)).to(dtype)
        s["residual"] = normal(rows, n_out).to(dtype) if case["residual"] else None
        s["y"] = torch.empty((rows, n_out), dtype=dtype, device="cuda")
        if case["train"]:
            # the backward pass takes the z that a forward pass left; drawn here, so that no rounding of z decides a slope
            s["dy"] = normal(rows, n_out).to(dtype)
            if case["act"] != "none":
                s["z"], s["z_out"] = (1.4 * normal(rows, n_out)).to(dtype), torch.empty_like(s["y"])
            s["dx"], s["dw"], s["dbias"] = torch.empty_like(s["x"]), torch.empty_like(s["w"]), torch.empty_like(s["bias"])
        return s
    classes, k = case["classes"], case["k"]
    # a network's logits: most classes far below a handful of likely ones; the last classes of a padded output are masked
    logits = normal(rows, classes) * 2.0
    likely = torch.randint(classes, (rows, 8), generator=g, device="cuda")
    logits.scatter_add_(1, likely, 6.0 + 2.0 * normal(rows, 8))
    logits[:, classes - classes // 100:] = float("-inf")
    seen = classes - classes // 100
    labels = torch.where(likely[:, 0] < seen, likely[:, 0], torch.randint(seen, (rows,), generator=g, device="cuda"))
    labels[5::16] = -1                                       # padding of the batch
    s["labels"] = labels.to(torch.int32)
    if case["op"] == "distill":
        teacher = logits + 0.5 * normal(rows, classes)
        top = teacher.topk(min(k, seen), dim=1)
        s["ids"] = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
        s["teacher"] = torch.zeros((rows, k), device="cuda")
        s["ids"][:, :min(k, seen)], s["teacher"][:, :min(k, seen)] = top.indices.to(torch.int32), top.values
        # the batch's mean; gradients in fp16 travel scaled up, as their users keep them from underflowing
        s["d_loss"] = (labels >= 0).float() * ((1024.0 if case["type"] == "fp16" else 1.0) / rows)
        s["loss"], s["stats"] = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    else:
        s["logprob"], s["entropy"], s["lse"] = (torch.empty(rows, device="cuda") for _ in range(3))
        s["top_ids"] = torch.empty((rows, k), dtype=torch.int32, device="cuda") if k else None
        s["top_logprobs"] = torch.empty((rows, k), device="cuda") if k else None
        s["d_logprob"], s["d_entropy"] = normal(rows), 0.1 * normal(rows)
    s["logits"] = logits.to(dtype)
    s["d_logits"] = torch.empty_like(s["logits"]) if case["op"] == "distill" or case["train"] else None
    return s


# ---- the operators in plain torch, 32 bits ---------------------------------------------------------------------------
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    sig = torch.sigmoid(z)
    return sig * (1.0 + z * (1.0 - sig))


def _plain_linear(s):
    case = s["case"]
    dtype = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.T + s["bias"].float()
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dtype)}
    if case["train"]:
        dz = s["dy"].float()
        if case["act"] != "none":
            dz = dz * _act_slope(s["z"].float(), case["act"])
            out["z"] = z.to(dtype)
        out.update(dx=(dz @ w).to(dtype), dw=(dz.T @ x).to(dtype), dbias=dz.sum(0).to(dtype))
    return out


def _log_softmax(v):
    """Rows of log-probabilities with their log-sum-exp; -inf stays -inf."""
    top = v.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(v - top).sum(1, keepdim=True))
    return v - lse, lse[:, 0]


def _plain_logprobs(s):
    case = s["case"]
    logp, lse = _log_softmax(s["logits"].float() / case["temperature"])
    p = torch.exp(logp)
    finite = torch.where(p > 0, logp, torch.zeros_like(logp))
    entropy = -(p * finite).sum(1)
    labels = s["labels"].long()
    there = labels >= 0
    at = labels.clamp_min(0)[:, None]
    logprob = torch.where(there, logp.gather(1, at)[:, 0], torch.zeros_like(lse))
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if case["k"]:
        # unique keys: the value's bits in their order, then the lower index first
        bits = s["logits"].float().view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        index = torch.arange(case["classes"], device="cuda")
        k = min(case["k"], case["classes"])
        ids = (order * (1 << 20) + ((1 << 20) - 1 - index)).topk(k, dim=1).indices
        values = logp.gather(1, ids)
        ids = torch.where(values > -math.inf, ids, torch.full_like(ids, -1))
        out["top_ids"] = torch.full((case["rows"], case["k"]), -1, dtype=torch.int32, device="cuda")
        out["top_logprobs"] = torch.full((case["rows"], case["k"]), -math.inf, device="cuda")
        out["top_ids"][:, :k], out["top_logprobs"][:, :k] = ids.to(torch.int32), values
    if case["train"]:
        g_lp = torch.where(there, s["d_logprob"], torch.zeros_like(lse))[:, None]
        d = -p * (g_lp + s["d_entropy"][:, None] * (finite + entropy[:, None]))
        d.scatter_add_(1, at, g_lp)
        out["d_logits"] = (d / case["temperature"]).to(s["logits"].dtype)
    return out


def _plain_distill(s):
    case = s["case"]
    T, alpha = case["temperature"], case["alpha"]
    v = s["logits"].float()
    ids, labels = s["ids"].long(), s["labels"].long()
    listed_ = ids >= 0
    q, _ = _log_softmax(torch.where(listed_, s["teacher"] / T, torch.full_like(s["teacher"], -math.inf)))
    logp, _ = _log_softmax(v / T)
    at = ids.clamp_min(0)
    weight = torch.exp(q)
    soft = torch.where(weight > 0, weight * (q - logp.gather(1, at)), torch.zeros_like(weight)).sum(1)
    loss = alpha * T * T * soft
    d = alpha * T * torch.exp(logp)
    d.scatter_add_(1, at, -alpha * T * weight)
    if alpha < 1:
        hard, _ = _log_softmax(v)
        there = (labels >= 0).float()
        label = labels.clamp_min(0)[:, None]
        loss = loss - (1 - alpha) * there * hard.gather(1, label)[:, 0]
        d = d + (1 - alpha) * there[:, None] * torch.exp(hard)
        d.scatter_add_(1, label, -(1 - alpha) * there[:, None])
    return {"loss": loss, "d_logits": (d * s["d_loss"][:, None]).to(s["logits"].dtype)}


# ---- the library's calls ---------------------------------------------------------------------------------------------
def _own_linear(s):
    import paper_1911_05146_b200 as hpf
    case = s["case"]
    rows, n_in, n_out = case["rows"], case["in"], case["out"]
    act = ACTS.index(case["act"])
    size = (rows, n_in, n_out, n_in, n_out)
    if "scratch" not in s:
        s["scratch"] = torch.zeros(hpf.linear_scratch_bytes(*size, s["x"].dtype, act), dtype=torch.uint8, device="cuda")
    hpf.linear_fwd(s["x"], s["w"], s["bias"], s["residual"], s["y"], s.get("z_out"), *size, act, s["scratch"])
    if not case["train"]:
        return {"y": s["y"]}
    hpf.linear_bwd(s["dy"], s.get("z"), s["x"], s["w"], s["dx"], s["dw"], s["dbias"], *size, act, s["scratch"])
    out = {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}
    return out if case["act"] == "none" else {**out, "z": s["z_out"]}


def _own_logprobs(s):
    import paper_1911_05146_b200 as hpf
    case = s["case"]
    rows, classes, k, T = case["rows"], case["classes"], case["k"], case["temperature"]
    hpf.logprobs_fwd(s["logits"], s["labels"], s["logprob"], s["entropy"], s["lse"], s["top_ids"], s["top_logprobs"], rows, classes, classes, k, T)
    out = {"logprob": s["logprob"], "entropy": s["entropy"], "lse": s["lse"]}
    if k:
        out.update(top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
    if case["train"]:
        hpf.logprobs_bwd(s["logits"], s["labels"], s["lse"], s["entropy"], s["d_logprob"], s["d_entropy"], s["d_logits"], rows, classes, classes, classes, T)
        out["d_logits"] = s["d_logits"]
    return out


def _own_distill(s):
    import paper_1911_05146_b200 as hpf
    case = s["case"]
    rows, classes, k, T, alpha = case["rows"], case["classes"], case["k"], case["temperature"], case["alpha"]
    if case["fused"]:
        hpf.distill_fwd_bwd(s["logits"], s["labels"], s["ids"], s["teacher"], s["d_loss"], s["loss"], s["d_logits"], rows, classes, classes, classes, k, T, alpha)
    else:
        hpf.distill_fwd(s["logits"], s["labels"], s["ids"], s["teacher"], s["loss"], s["stats"], rows, classes, classes, k, T, alpha)
        hpf.distill_bwd(s["logits"], s["labels"], s["ids"], s["teacher"], s["stats"], s["d_loss"], s["d_logits"], rows, classes, classes, classes, k, T, alpha)
    return {"loss": s["loss"], "d_logits": s["d_logits"]}


def run(s):
    op = s["case"]["op"]
    if op == "linear":
        return _own_linear(s) if own else _plain_linear(s)
    if op == "logprobs":
        return _own_logprobs(s) if own else _plain_logprobs(s)
    return _own_distill(s) if own else _plain_distill(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    e = 4.0 if case["type"] == "fp32" else 2.0
    rows = case["rows"]
    if case["op"] == "linear":
        n_in, n_out = case["in"], case["out"]
        values = rows * n_in + n_out * n_in + n_out + rows * n_out * (2 if case["residual"] else 1)
        if case["train"]:
            values += rows * n_out + rows * n_in + n_out * n_in + n_out      # dy read, dx, dW and db written
            values += 2 * rows * n_out if case["act"] != "none" else 0       # z written, z read
        return {"bytes": e * values, "flops": 2.0 * rows * n_in * n_out * (3 if case["train"] else 1)}
    n = float(rows) * case["classes"]
    if case["op"] == "logprobs":
        back = case["train"]
        return {"bytes": e * n * (3 if back else 1) + rows * (16.0 + 8.0 * case["k"] + (20.0 if back else 0.0)), "flops": n * (12.0 if back else 5.0)}
    return {"bytes": e * n * (2 if case["fused"] else 3) + rows * (12.0 + 8.0 * case["k"]), "flops": n * (14.0 if case["alpha"] < 1 else 8.0)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, s)
    return _exact_logprobs(case, s) if case["op"] == "logprobs" else _exact_distill(case, s)


def _exact_linear(case, s):
    x, w = s["x"].double(), s["w"].double()
    z = torch.addmm(s["bias"].double(), x, w.t())
    out = {"y": _exact_value(z, case["act"])}
    if case["residual"]:
        out["y"] += s["residual"].double()
    if case["train"]:
        dz = s["dy"].double()
        if case["act"] != "none":
            out["z"] = z
            dz = dz * _exact_derivative(s["z"].double(), case["act"])
        out.update(dx=torch.mm(dz, w), dw=torch.mm(dz.t(), x), dbias=dz.sum(dim=0))
    return out


def _exact_cdf(z, act):
    """What gelu and silu multiply z with."""
    return 0.5 * torch.erfc(-z / math.sqrt(2.0)) if act == "gelu" else 1.0 / (1.0 + torch.exp(-z))


def _exact_value(z, act):
    if act == "none":
        return z.clone()
    return torch.where(z > 0, z, 0.0) if act == "relu" else z * _exact_cdf(z, act)


def _exact_derivative(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    c = _exact_cdf(z, act)
    return c + z * (torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if act == "gelu" else c * (1 - c))


def _exact_logprobs(case, s):
    v = s["logits"].double() / case["temperature"]
    rows = torch.arange(case["rows"], device=v.device)
    labels = s["labels"].long()
    there = (labels >= 0).double()
    lse = torch.logsumexp(v, 1)
    logp = v - lse[:, None]
    p = torch.softmax(v, 1)
    entropy = torch.special.entr(p).sum(1)
    out = {"logprob": torch.where(labels >= 0, logp[rows, labels.clamp(min=0)], 0.0), "entropy": entropy, "lse": lse}
    if case["k"]:
        k = min(case["k"], case["classes"])
        best = torch.full((case["rows"], case["k"]), -math.inf, dtype=torch.float64, device=v.device)
        best[:, :k] = torch.topk(logp, k, 1).values
        out.update(top_ids=None, top_logprobs=best)
    if case["train"]:
        g, h = s["d_logprob"].double() * there, s["d_entropy"].double()
        d = -g[:, None] * p + h[:, None] * (torch.special.entr(p) - p * entropy[:, None])
        d[rows, labels.clamp(min=0)] += g
        out["d_logits"] = d / case["temperature"]
    return out


def _exact_distill(case, s):
    T, alpha = case["temperature"], case["alpha"]
    v = s["logits"].double()
    rows = torch.arange(case["rows"], device=v.device)
    target = torch.zeros_like(v)
    ids = s["ids"].long()
    q = torch.softmax(s["teacher"].double().masked_fill(ids < 0, -math.inf) / T, 1)
    target.scatter_add_(1, ids.clamp(min=0), q)
    d = alpha * T * (torch.softmax(v / T, 1) - target)
    chosen = torch.log_softmax(v / T, 1).gather(1, ids.clamp(min=0))
    loss = alpha * T * T * (-torch.special.entr(q) - torch.where(q > 0, q * chosen, 0.0)).sum(1)
    if alpha < 1:
        labels = s["labels"].long()
        there = (labels >= 0).double() * (1 - alpha)
        h = torch.softmax(v, 1)
        loss = loss + there * (torch.logsumexp(v, 1) - v[rows, labels.clamp(min=0)])
        h[rows, labels.clamp(min=0)] -= 1.0
        d = d + there[:, None] * h
    return {"loss": loss, "d_logits": d * s["d_loss"].double()[:, None]}
