"""The linear layer, log-probabilities and distillation together, as a training loop uses them: a teacher writes down its likeliest classes, a
student learns from the list and the labels over micro-batches whose gradients go into flat fp32 slots, and the update ends the step."""
import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, F, C, K, M, T, ALPHA, LR, MU, WD = 96, 128, 1000, 16, 2, 2.0, 0.6, 0.1, 0.9, 1e-4


class Step:
    """Weights of type `dtype` to multiply with, the student's masters in fp32 (the same buffer where dtype is fp32)."""

    def __init__(self, dtype, seed=0):
        g = torch.Generator(device=DEV); g.manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.dtype, e = dtype, lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)
        self.x = normal(B, F).to(dtype)
        self.labels = torch.randint(C, (B,), generator=g, device=DEV, dtype=torch.int32)
        self.labels[::7] = -1
        self.wt, self.bt = (2.0 * normal(C, F) / F ** 0.5).to(dtype), (0.1 * normal(C)).to(dtype)
        self.params = torch.cat([normal(C * F) / F ** 0.5, 0.1 * normal(C)])
        self.velocity, self.avg, self.slots = e(C * F + C), e(C * F + C), e(M, C * F + C)
        self.w, self.b = self._weights()
        self.t_logits, self.logits = e(B, C, t=dtype), e(B, C, t=dtype)
        self.ids, self.top, self.loss = e(B, K, t=torch.int32), e(B, K), e(B)
        self.weight = torch.full((B,), M / B, device=DEV)
        self.scratch = torch.zeros(hpf.linear_scratch_bytes(B, F, C, F, C, dtype), dtype=torch.uint8, device=DEV)

    def _weights(self):
        w, b = self.params[:C * F].view(C, F), self.params[C * F:]
        return (w, b) if self.dtype == torch.float32 else (w.to(self.dtype), b.to(self.dtype))

    def run(self):
        size = (B, F, C, F, C, hpf.ACT_NONE, self.scratch)
        hpf.linear_fwd(self.x, self.wt, self.bt, None, self.t_logits, None, *size)
        hpf.logprobs_fwd(self.t_logits, None, None, None, None, self.ids, self.top, B, C, C, K)
        hpf.linear_fwd(self.x, self.w, self.b, None, self.logits, None, *size)
        # the gradient takes the logits' place
        hpf.distill_fwd_bwd(self.logits, self.labels, self.ids, self.top, self.weight, self.loss, self.logits, B, C, C, C, K, T, ALPHA)
        for m in range(M):
            rows = slice(m * B // M, (m + 1) * B // M)
            slot = self.slots[m]
            hpf.linear_bwd(self.logits[rows], None, self.x[rows], self.w, None, slot[:C * F].view(C, F), slot[C * F:], B // M, *size[1:])
        hpf.sgd_momentum_flat(self.slots, self.avg, self.params, self.velocity, M, C * F + C, LR, MU, WD)
        if self.dtype != torch.float32:
            self.w.copy_(self.params[:C * F].view(C, F))
            self.b.copy_(self.params[C * F:])


def test_a_step_in_fp32_against_64_bits():
    s = Step(torch.float32)
    x, wt, bt, labels = s.x.double(), s.wt.double(), s.bt.double(), s.labels.long()
    w0, p0 = s.params[:C * F].view(C, F).double().clone(), s.params.double().clone()
    s.run()
    torch.cuda.synchronize()
    # logits are within tau of their definition: 3 2^-20 of the magnitudes that are summed up (see test_gpu_linear), and the additions' 2^-23
    teacher, student = x @ wt.T + bt, x @ w0.T + p0[C * F:]
    tau = 4 * 2.0 ** -20 * max((x.abs() @ wt.abs().T).max().item(), (x.abs() @ w0.abs().T).max().item())
    ids = s.ids.long()
    listed = teacher.gather(1, ids)
    rest = teacher.scatter(1, ids, float("-inf")).amax(1)
    assert (listed.amin(1) >= rest - 2 * tau).all() and (listed[:, :-1] >= listed[:, 1:] - 2 * tau).all()
    q = torch.softmax(listed / T, 1)
    lp, hard = torch.log_softmax(student / T, 1), torch.log_softmax(student, 1)
    there = (labels >= 0).double()
    at = labels.clamp_min(0)[:, None]
    loss = ALPHA * T * T * (q * (q.log() - lp.gather(1, ids))).sum(1) - (1 - ALPHA) * there * hard.gather(1, at)[:, 0]
    # every logarithm is off by at most 2 tau, q's share of it likewise
    assert ((s.loss.double() - loss).abs() <= (ALPHA * T * T * 4 / T + 2) * tau + 1e-4).all()
    d = ALPHA * T * lp.exp() + (1 - ALPHA) * there[:, None] * hard.exp()
    off = d * 4 * tau + 1e-6
    d.scatter_add_(1, ids, -ALPHA * T * q)
    off.scatter_add_(1, ids, ALPHA * T * q * 4 * tau)
    d.scatter_add_(1, at, -(1 - ALPHA) * there[:, None])
    d, off = d * M / B, off * M / B
    grad = torch.cat([(d.T @ x).flatten(), d.sum(0)]) / M
    tol = torch.cat([(off.T @ x.abs() + 4 * 2.0 ** -20 * (d.abs().T @ x.abs())).flatten(), off.sum(0) + 2.0 ** -20 * d.abs().sum(0)]) / M
    assert ((s.avg.double() - grad).abs() <= tol + 1e-9).all()
    v = -LR * (grad + WD * p0)
    assert ((s.params.double() - (p0 + v)).abs() <= LR * tol + 2.0 ** -23 * p0.abs() + 1e-9).all()
    assert not hpf.linear_status(s.scratch)


def test_a_step_in_bf16_leaves_fp32_gradients():
    """The products of two bf16 values are exact in fp32: the slots are off by their sums' rounding alone."""
    s = Step(torch.bfloat16)
    s.run()
    torch.cuda.synchronize()
    for m in range(M):
        rows = slice(m * B // M, (m + 1) * B // M)
        d, x = s.logits[rows].double(), s.x[rows].double()
        for got, want, size in ((s.slots[m, :C * F].view(C, F), d.T @ x, d.abs().T @ x.abs()), (s.slots[m, C * F:], d.sum(0), d.abs().sum(0))):
            assert ((got.double() - want).abs() <= size * 40 * 2.0 ** -23 + 1e-12).all()
    assert torch.equal(s.w, s.params[:C * F].view(C, F).bfloat16())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_step_in_a_graph_gives_the_same_bits(dtype):
    eager, graphed = Step(dtype), Step(dtype)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.run()
    for _ in range(3):
        eager.run()
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(eager.params, graphed.params) and torch.equal(eager.loss, graphed.loss) and torch.equal(eager.ids, graphed.ids)
    assert torch.isfinite(eager.params).all() and not torch.equal(eager.params, Step(dtype).params)


def test_two_threads_at_once():
    """Each with its own stream, buffers and scratch; the calls leave the interpreter's lock while they launch."""
    steps = [Step(torch.bfloat16, seed) for seed in (1, 2)]
    alone = [Step(torch.bfloat16, seed) for seed in (1, 2)]
    for s in alone:
        for _ in range(10):
            s.run()
    torch.cuda.synchronize()
    failed = []

    def work(s, stream):
        try:
            with torch.cuda.stream(stream):
                for _ in range(10):
                    s.run()
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=work, args=(s, torch.cuda.Stream())) for s in steps]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    assert all(torch.equal(a.params, b.params) for a, b in zip(steps, alone))


def test_the_first_calls_of_a_process_may_be_captured():
    """Whatever a call sets up once, it can set up inside a capture."""
    here = os.path.dirname(os.path.abspath(__file__))
    code = ("import sys, torch\n"
            f"sys.path[:0] = [{os.path.dirname(here)!r}, {here!r}]\n"
            "import test_gpu_distillation_run as t\n"
            "s = t.Step(torch.bfloat16); e = t.Step(torch.bfloat16)\n"
            "torch.cuda.synchronize()\n"
            "g = torch.cuda.CUDAGraph()\n"
            "with torch.cuda.graph(g):\n"
            "    s.run()\n"
            "g.replay(); e.run(); torch.cuda.synchronize()\n"
            "assert torch.equal(s.params, e.params) and torch.equal(s.loss, e.loss)\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
