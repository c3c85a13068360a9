"""The linear layer on the GPU against its formulas in 64 bits.

Tolerances.  A sum of K products is off by at most one step of fp32 (2^-23) of the sum of magnitudes A = sum |x| |w| per addition into the accumulator,
which truncates: K / 16 additions with 16-bit operands (K / 8 times three with fp32 ones, counted from anew every 128 bytes of k times 4, so 48 and one
rounding per such chunk), twice that for what one instruction adds up inside.  fp32 products miss 3 2^-20 of their magnitude.  An activation
passes errors on with a factor below 1.2 and adds a few 2^-23 of |z|.  Every rounding to the tensor's type is half a step, eps / 2, of the value (fp16: or
half its smallest step, 2^-25).  dz is rounded once before it enters dx and dW where there is an activation.
"""
import math

import pytest
import torch

import paper_1911_05146_b200 as hpf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def act64(z, act):
    if act == hpf.ACT_RELU:
        return z.clamp_min(0)
    if act == hpf.ACT_GELU:
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    return z * torch.sigmoid(z) if act == hpf.ACT_SILU else z


def slope64(z, act):
    if act == hpf.ACT_RELU:
        return (z > 0).double()
    if act == hpf.ACT_GELU:
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s)) if act == hpf.ACT_SILU else torch.ones_like(z)


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _sum_tol(K, magnitude, dtype, out):
    """error of a product's sums before the last rounding"""
    if dtype == torch.float32:
        return magnitude * (3 * 2.0 ** -20 + (2 * 48 + K / 128) * 2.0 ** -23)
    if out == torch.float32:
        return magnitude * ((2 * 16 + K / 256) * 2.0 ** -23)
    return magnitude * (2 * (K / 16 + 2) * 2.0 ** -23)


def _within(got, want, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    least = 2.0 ** -25
    off = ((got - want).abs() / (tol + least)).max().item()
    assert off <= 1.0, (what, off)


class Case:
    def __init__(self, rows, n_in, n_out, dtype, act, *, gap_x=0, gap_y=0, offset=0, residual=True, bias=True, seed=0):
        t = self.t = TYPES[dtype]
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + 7 * rows + 13 * n_in + 17 * n_out)
        self.size = (rows, n_in, n_out, n_in + gap_x, n_out + gap_y)
        self.act, self.rows, self.n_in, self.n_out = act, rows, n_in, n_out

        def rowed(n, gap, fill):
            """rows of n values, `gap` apart, starting `offset` values into a buffer of NaNs (nothing between rows may be read into a sum)"""
            buf = torch.full((offset + rows * (n + gap),), float("nan"), dtype=t, device=DEV)
            v = buf[offset:].as_strided((rows, n), (n + gap, 1))
            if fill is not None:
                v.copy_(fill)
            return v
        normal = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.x = rowed(n_in, gap_x, normal(rows, n_in))
        wbuf = torch.empty(offset + n_out * n_in, dtype=t, device=DEV)
        self.w = wbuf[offset:].view(n_out, n_in)
        self.w.copy_(normal(n_out, n_in) * math.sqrt(2.0 / n_in))
        self.bias = (0.3 * normal(n_out)).to(t) if bias else None
        self.residual = rowed(n_out, gap_y, normal(rows, n_out)) if residual else None
        self.dy = rowed(n_out, gap_y, normal(rows, n_out))
        self.z = rowed(n_out, gap_y, 1.3 * normal(rows, n_out))
        self.y, self.z_out = rowed(n_out, gap_y, None), rowed(n_out, gap_y, None)
        self.dx = rowed(n_in, gap_x, None)
        self.scratch = torch.zeros(hpf.linear_scratch_bytes(*self.size, t, act, aligned=offset == 0), dtype=torch.uint8, device=DEV)

    def forward(self, y=None, residual="own", stream=None):
        res = self.residual if residual == "own" else residual
        hpf.linear_fwd(self.x, self.w, self.bias, res, self.y if y is None else y, self.z_out, *self.size, self.act, self.scratch, stream)

    def backward(self, grad=None, want=("dx", "dw", "db")):
        g = grad or self.t
        self.dw = torch.full((self.n_out, self.n_in), float("nan"), dtype=g, device=DEV)
        self.db = torch.full((self.n_out,), float("nan"), dtype=g, device=DEV)
        hpf.linear_bwd(self.dy, self.z if self.act else None, self.x, self.w, self.dx if "dx" in want else None, self.dw if "dw" in want else None,
                       self.db if "db" in want else None, *self.size, self.act, self.scratch)

    def check_forward(self):
        x, w = self.x.double(), self.w.double()
        b = self.bias.double() if self.bias is not None else torch.zeros(self.n_out, dtype=torch.float64, device=DEV)
        z = x @ w.T + b
        zt = _sum_tol(self.n_in, x.abs() @ w.abs().T, self.t, self.t) + 2.0 ** -23 * (z.abs() + b.abs())
        _within(self.z_out, z, zt + _half(self.t) * z.abs(), "z")
        y = act64(z, self.act)
        r = self.residual.double() if self.residual is not None else 0 * y
        _within(self.y, y + r, 1.2 * zt + 2.0 ** -21 * z.abs() + 2.0 ** -23 * (y.abs() + r.abs()) + _half(self.t) * (y + r).abs(), "y")
        assert not hpf.linear_status(self.scratch)

    def check_backward(self, grad=None):
        g = grad or self.t
        x, w, z = self.x.double(), self.w.double(), self.z.double()
        dz = self.dy.double() * slope64(z, self.act)
        one = 0.0 if not self.act else _half(self.t) + 2.0 ** -20          # dz: its rounding and its slope's few 2^-23 (of 1 + |z|)
        dzt = one * dz.abs() + (2.0 ** -21 * self.dy.double().abs() * (1 + z.abs()) if self.act else 0 * dz)
        dzt = dzt + (2.0 ** -25 if self.t == torch.float16 and self.act else 0.0)
        dx = dz @ w
        _within(self.dx, dx, _sum_tol(self.n_out, dz.abs() @ w.abs(), self.t, self.t) + dzt @ w.abs() + _half(self.t) * dx.abs(), "dx")
        dw = dz.T @ x
        _within(self.dw, dw, _sum_tol(self.rows, dz.abs().T @ x.abs(), self.t, g) + dzt.T @ x.abs() + _half(g) * dw.abs(), "dw")
        db = dz.sum(0)
        adds = self.rows / 32 + 32
        _within(self.db, db, dz.abs().sum(0) * adds * 2.0 ** -24 + (2.0 ** -21 * (self.dy.double().abs() * (1 + z.abs())).sum(0) if self.act else 0.0) + _half(g) * db.abs(), "db")
        assert not hpf.linear_status(self.scratch)


# single rows, odd sizes, one tile to several per CTA, long k split over a cluster, k below one stage
SHAPES = [(1, 16, 10), (1, 2048, 512), (2, 1, 1), (3, 27, 33), (17, 8, 4100), (64, 2048, 1000), (129, 513, 257), (128, 64, 64), (128, 4096, 256), (300, 1000, 130),
          (257, 96, 300), (1000, 129, 1025), (2600, 136, 4104)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n_in, n_out", SHAPES)
def test_forward_and_gradients(rows, n_in, n_out, dtype):
    act = (rows + n_in) % 4
    c = Case(rows, n_in, n_out, dtype, act)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", [0, 1, 2, 3])
def test_every_activation(act, dtype):
    for residual, bias in ((True, False), (False, True)):
        c = Case(200, 160, 96, dtype, act, residual=residual, bias=bias, seed=act)
        c.forward()
        c.backward()
        torch.cuda.synchronize()
        c.check_forward()
        c.check_backward()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gap_x, gap_y, offset", [(8, 16, 0), (3, 0, 0), (0, 5, 0), (0, 0, 1), (1, 1, 3)])
@pytest.mark.parametrize("rows, n_in, n_out, act", [(70, 136, 72, 2), (5, 45, 77, 0), (140, 64, 200, 0)])
def test_strides_and_alignments(rows, n_in, n_out, act, gap_x, gap_y, offset, dtype):
    """Rows apart, off 16-byte boundaries and off the start of their buffers; what lies between rows is neither read nor written."""
    c = Case(rows, n_in, n_out, dtype, act, gap_x=gap_x, gap_y=gap_y, offset=offset)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    c.check_forward()
    c.check_backward()
    for v, n, gap in ((c.y, n_out, gap_y), (c.z_out, n_out, gap_y), (c.dx, n_in, gap_x)):
        if gap:
            between = v.as_strided((rows - 1, gap), (n + gap, 1), v.storage_offset() + n)
            assert torch.isnan(between).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows, n_in, n_out, act", [(1, 40, 50, 0), (700, 130, 140, 0), (1500, 256, 64, 3)])
def test_weight_gradients_in_fp32(rows, n_in, n_out, act, dtype):
    """The form that the fp32 gradient slots take."""
    c = Case(rows, n_in, n_out, dtype, act)
    c.backward(grad=torch.float32)
    torch.cuda.synchronize()
    c.check_backward(grad=torch.float32)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_each_gradient_alone_is_the_same(dtype):
    c = Case(150, 72, 90, dtype, hpf.ACT_SILU)
    c.backward()
    whole = [t.clone() for t in (c.dx, c.dw, c.db)]
    for i, name in enumerate(("dx", "dw", "db")):
        c.dx.fill_(float("nan"))
        c.backward(want=(name,))
        torch.cuda.synchronize()
        assert torch.equal((c.dx, c.dw, c.db)[i], whole[i])
        assert all(torch.isnan(t).all() for j, t in enumerate((c.dx, c.dw, c.db)) if j != i)


def test_gradients_against_differences():
    """Directional differences of the forward call: the loss is sum(dy * y), its derivative along (u, v, t) is <dx, u> + <dW, v> + <db, t>."""
    c = Case(40, 48, 56, "fp32", hpf.ACT_GELU, residual=False)
    h = 2.0 ** -7
    c.forward()
    c.z.copy_(c.z_out)
    c.backward()
    x, w, b = c.x.clone(), c.w.clone(), c.bias.clone()
    g = torch.Generator(device=DEV); g.manual_seed(3)
    u, v, t = (torch.randn(s.shape, generator=g, device=DEV) for s in (x, w, b))
    v *= 0.1
    ends = []
    for sign in (1, -1):
        c.x.copy_(x + sign * h * u); c.w.copy_(w + sign * h * v); c.bias.copy_(b + sign * h * t)
        c.forward()
        ends.append((c.dy.double() * c.y.double()).sum().item())
    slope = (c.dx.double() * u).sum() + (c.dw.double() * v).sum() + (c.db.double() * t).sum()
    # along the line z moves by h s with |s| up to about 30 (48 products of variance near 1 / 4 and 2, and the cross term): h^2 / 6 times a third
    # derivative below 1.2 |s|^3 + 3 |u v| terms, random in sign over 2240 outputs of dy near 1: well under 0.01 of the slope's own scale
    scale = math.sqrt(sum(((a.double() * d.double()) ** 2).sum().item() for a, d in ((c.dx, u), (c.dw, v), (c.db, t))))
    assert abs((ends[0] - ends[1]) / (2 * h) - slope.item()) <= 0.05 * scale


def test_residual_may_be_the_output():
    c = Case(133, 80, 104, "bf16", hpf.ACT_RELU)
    c.forward()
    y = c.residual.clone()
    hpf.linear_fwd(c.x, c.w, c.bias, y, y, None, *c.size, c.act, c.scratch)
    torch.cuda.synchronize()
    assert torch.equal(y, c.y)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, n_in, n_out", [(1, 4096, 320), (100, 2048, 128), (900, 320, 640)])
def test_repeats_streams_and_graphs_give_the_same_bits(rows, n_in, n_out, dtype):
    c = Case(rows, n_in, n_out, dtype, hpf.ACT_GELU)

    def both():
        c.forward()
        c.backward()
        return [t.clone() for t in (c.y, c.z_out, c.dx, c.dw, c.db)]
    first = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward()
        c.backward()
    graphed = (c.y, c.z_out, c.dx, c.dw, c.db)
    c.x.mul_(2.0)
    g.replay()
    torch.cuda.synchronize()
    third = [t.clone() for t in graphed]
    assert all(torch.equal(a, b) for a, b in zip(third, both()))
    assert not torch.equal(third[0], first[0])


def test_two_streams_at_once():
    """Calls that overlap, each with a scratch of its own."""
    cases = [Case(500, 256, 300, "bf16", 2, seed=i) for i in range(2)] + [Case(100, 1024, 200, "fp32", 3, seed=i) for i in range(2)]
    alone = []
    for c in cases:
        c.forward(); c.backward()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (c.y, c.dx, c.dw, c.db)])
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[] for _ in cases]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                c.forward(); c.backward()
                outs[i].append([t.clone() for t in (c.y, c.dx, c.dw, c.db)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, o in enumerate(outs) for r in o for a, b in zip(r, alone[i]))


def test_an_empty_batch():
    t = torch.bfloat16
    e = lambda *s: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
    dw, db = torch.full((4, 8), 3.0, device=DEV), torch.full((4,), 3.0, device=DEV)
    scratch = torch.zeros(256, dtype=torch.uint8, device=DEV)
    hpf.linear_fwd(e(0, 8), e(4, 8), None, None, e(0, 4), None, 0, 8, 4, 8, 4, 0, scratch)
    hpf.linear_bwd(e(0, 4), None, e(0, 8), e(4, 8), e(0, 8), dw, db, 0, 8, 4, 8, 4, 0, scratch)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()


def test_infinities_and_nans_stay_in_their_rows():
    c = Case(140, 64, 96, "bf16", hpf.ACT_NONE)
    c.x[3, 5] = float("inf")
    c.x[130, 1] = float("nan")
    c.forward()
    torch.cuda.synchronize()
    bad = torch.zeros(140, dtype=torch.bool, device=DEV)
    bad[3] = bad[130] = True
    assert torch.isfinite(c.y[~bad]).all() and not torch.isfinite(c.y[bad]).any()


def test_binding_refuses_what_the_kernels_would_misread():
    c = Case(4, 16, 24, "bf16", 0)
    with pytest.raises(hpf.HpfError):
        hpf.linear_fwd(c.x, c.w.float(), None, None, c.y, None, *c.size, 0, c.scratch)
    with pytest.raises(hpf.HpfError):
        hpf.linear_fwd(c.x.cpu(), c.w, None, None, c.y, None, *c.size, 0, c.scratch)
    with pytest.raises(hpf.HpfError):
        hpf.linear_fwd(c.x, c.w, None, None, c.y, None, *c.size, 0, c.scratch[:100])
    with pytest.raises(hpf.HpfError):
        hpf.linear_bwd(c.dy, None, c.x, c.w, c.dx, torch.zeros((24, 16), dtype=torch.float16, device=DEV), None, *c.size, 0, c.scratch)


def test_offsets_beyond_32_bits():
    """Rows that start more than 2^32 elements into their buffers."""
    rows, n_in, n_out, ld = 3, 40, 72, (1 << 31) + 8
    t = torch.bfloat16
    x, dx, y, dy = (torch.empty((rows - 1) * ld + n, dtype=t, device=DEV).as_strided((rows, n), (ld, 1)) for n in (n_in, n_in, n_out, n_out))
    g = torch.Generator(device=DEV); g.manual_seed(1)
    x.copy_(torch.randn(rows, n_in, generator=g, device=DEV)); dy.copy_(torch.randn(rows, n_out, generator=g, device=DEV))
    w = torch.randn(n_out, n_in, generator=g, device=DEV).to(t)
    dw, db = torch.empty_like(w), torch.empty(n_out, dtype=t, device=DEV)
    size = (rows, n_in, n_out, ld, ld, hpf.ACT_NONE)
    scratch = torch.zeros(hpf.linear_scratch_bytes(*size[:5], t), dtype=torch.uint8, device=DEV)
    hpf.linear_fwd(x, w, None, None, y, None, *size, scratch)
    hpf.linear_bwd(dy, None, x, w, dx, dw, db, *size, scratch)
    torch.cuda.synchronize()
    X, W, D = x.double(), w.double(), dy.double()
    for got, want, size_ in ((y, X @ W.T, X.abs() @ W.abs().T), (dx, D @ W, D.abs() @ W.abs()), (dw, D.T @ X, D.abs().T @ X.abs()), (db, D.sum(0), D.abs().sum(0))):
        _within(got, want, _half(t) * want.abs() + 2.0 ** -20 * size_, "offsets")


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_behind_the_last_are_left_alone(dtype):
    """y, z and dx larger than the batch: what lies behind its last row stays as it was."""
    rows, n_in, n_out, more = 130, 64, 96, 3
    c = Case(rows, n_in, n_out, dtype, hpf.ACT_GELU)
    y, z, dx = (torch.full((rows + more, n), 5.0, dtype=c.t, device=DEV) for n in (n_out, n_out, n_in))
    hpf.linear_fwd(c.x, c.w, c.bias, c.residual, y, z, *c.size, c.act, c.scratch)
    hpf.linear_bwd(c.dy, c.z, c.x, c.w, dx, None, None, *c.size, c.act, c.scratch)
    c.forward(); c.backward()
    torch.cuda.synchronize()
    for big, small in ((y, c.y), (z, c.z_out), (dx, c.dx)):
        assert torch.equal(big[:rows], small) and (big[rows:] == 5.0).all()
