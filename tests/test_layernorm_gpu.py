"""Layer norm and its gradients against the formulas in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, half a step of fp32; `half` = half a step of the stored type).  Sums of n terms are
formed from at most 32 terms in a row (n / 1024 beyond 32768 columns), then pairwise over at most 10 levels: relative error of a sum of
non-negative terms below `chain` = (42 + n / 1024) u, of any sum that much of the sum of magnitudes.
  mean   chain * mean|x| + u |mean|
  rstd   the deviations inherit the mean's error e, which adds e^2 to the variance (the linear term sums to nothing but for chain
         * var), their own rounding 2 u and the squares' chain: relative error of var below 2 chain + (e / sigma)^2 + 4 u
         (|mean| / sigma) for the subtraction's rounding, of rstd half of that + 3 u
  y      with h = (x - mean) rstd: |h| times rstd's error + rstd (mean's error + u |x - mean|), 4 u of each of the terms h w and b,
         and `half` of y
  dx     rstd (d - c1 - h c2): 6 u of each term's magnitude, chain of the means' magnitudes, and `half` of dx
  sums   over rows: at most rows / (a block's share) + 64 terms one after another: (rows / 148 + 64) u of the sum of magnitudes,
         and each term's own 6 u."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SENT = -7.25


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _dt(torch, name):
    return torch.float32 if name == "f32" else torch.bfloat16


class Arena:
    """Matrices with a stride and an offset inside buffers whose other elements must stay."""

    def __init__(self, torch):
        self.torch, self.all = torch, []

    def matrix(self, rows, cols, ld, offset, dtype):
        flat = self.torch.full((64 + offset + rows * ld + 64,), SENT, dtype=_dt(self.torch, dtype), device="cuda")
        view = flat[64 + offset:64 + offset + rows * ld].view(rows, ld)[:, :cols]
        mask = self.torch.ones_like(flat, dtype=self.torch.bool)
        mask[64 + offset:64 + offset + rows * ld].view(rows, ld)[:, :cols] = False
        self.all.append((flat, mask))
        return view

    def intact(self):
        return all(bool((flat[mask] == SENT).all()) for flat, mask in self.all)


def _inputs(torch, a, rows, cols, ld, offset, dtype, wdt, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x = a.matrix(rows, cols, ld, offset, dtype)
    x.copy_(new(rows, cols) * torch.exp(new(rows, 1)) + 3 * new(rows, 1))
    w = new(cols).to(_dt(torch, wdt))
    b = new(cols).to(_dt(torch, wdt))
    return x, w, b, new


def _chain(cols):
    return (42 + cols / 1024) * U


def _check_forward(torch, x, w, b, eps, y, mean, rstd, out):
    cols = x.shape[1]
    x64 = x.double()
    mu, var = x64.mean(1, keepdim=True), x64.var(1, unbiased=False, keepdim=True)
    rs = (var + eps) ** -0.5
    dev = x64 - mu
    e_mean = _chain(cols) * x64.abs().mean(1, keepdim=True) + U * mu.abs()
    sigma = (var + eps).sqrt()
    # (the subtraction x - mean rounds by u of the deviation; its share of the variance stays below 2 u)
    e_var = 2 * _chain(cols) + (e_mean / sigma) ** 2 + 4 * U
    e_rstd = e_var / 2 + 3 * U
    if mean is not None:
        assert bool(((mean.double()[:, None] - mu).abs() <= e_mean + 1e-40).all())
        assert bool(((rstd.double()[:, None] - rs).abs() <= rs * e_rstd).all())
    h = dev * rs
    wd = w.double() if w is not None else torch.ones(cols, dtype=torch.float64, device="cuda")
    bd = b.double() if b is not None else torch.zeros(cols, dtype=torch.float64, device="cuda")
    want = h * wd + bd
    tol = (h.abs() * (e_rstd + 4 * U) + rs * e_mean) * wd.abs() + 4 * U * bd.abs() + HALF[out] * want.abs() * (1 + 1e-6)
    tol = tol * (1 + HALF[out]) + 1e-40
    assert bool(((y.double() - want).abs() <= tol).all()), float(((y.double() - want).abs() / tol).max())


SHAPES = [
    # rows, cols, extra stride, offset
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 0, 1), (2, 31, 2, 0), (4, 33, 0, 0), (1, 255, 0, 3), (17, 256, 0, 0), (9, 264, 8, 8), (300, 100, 0, 0),
    (7, 771, 0, 0), (40, 1000, 0, 0), (33, 1024, 0, 0), (301, 1032, 0, 0), (8, 4096, 0, 0), (299, 4096, 64, 0), (5, 5001, 0, 0), (3, 8192, 0, 0),
    (320, 8192, 0, 0), (2, 8200, 0, 0), (3, 16384, 0, 0), (2, 20001, 0, 0), (2, 32768, 0, 0), (301, 32776, 0, 0), (2, 70002, 0, 0), (1, 100001, 5, 1),
]


@pytest.mark.parametrize("rows,cols,extra,offset", SHAPES)
@pytest.mark.parametrize("dtype,out,wdt,affine", [("f32", "f32", "f32", "both"), ("bf16", "bf16", "f32", "both"), ("bf16", "f32", "bf16", "weight"),
                                                  ("f32", "bf16", "bf16", "bias"), ("bf16", "bf16", "bf16", "none")])
def test_forward(env, rows, cols, extra, offset, dtype, out, wdt, affine):
    torch, binding = env
    a = Arena(torch)
    x, w, b, _ = _inputs(torch, a, rows, cols, cols + extra, offset, dtype, wdt, 5)
    w, b = w if affine in ("both", "weight") else None, b if affine in ("both", "bias") else None
    y = a.matrix(rows, cols, cols + extra, offset, out)
    got, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-5, out=y)
    assert got is y and mean.shape == rstd.shape == (rows,)
    _check_forward(torch, x, w, b, 1e-5, y, mean, rstd, out)
    assert a.intact()
    alone = binding.layer_norm_forward(x, w, b, 1e-5, out_dtype=_dt(torch, out), stats=False)
    assert torch.equal(alone, y)


@pytest.mark.parametrize("rows,cols,extra,offset", SHAPES)
@pytest.mark.parametrize("dtype,gdt,out,wdt,add", [("f32", "f32", "f32", "f32", True), ("bf16", "bf16", "bf16", "f32", False), ("bf16", "f32", "bf16", "bf16", True),
                                                   ("f32", "bf16", "f32", "bf16", False)])
def test_backward(env, rows, cols, extra, offset, dtype, gdt, out, wdt, add):
    torch, binding = env
    a = Arena(torch)
    x, w, _, new = _inputs(torch, a, rows, cols, cols + extra, offset, dtype, wdt, 6)
    dy, dx = a.matrix(rows, cols, cols + extra, offset, gdt), a.matrix(rows, cols, cols + extra, offset, out)
    dy.copy_(new(rows, cols))
    mean, rstd = x.double().mean(1).float(), ((x.double().var(1, unbiased=False) + 1e-5) ** -0.5).float()
    dw, db = a.matrix(1, cols, cols, offset, wdt)[0], a.matrix(1, cols, cols, offset, wdt)[0]
    dw.copy_(new(cols))
    db.copy_(new(cols))
    old_w, old_b = dw.double(), db.double()
    got = binding.layer_norm_backward(dy, x, mean, rstd, w, grad_x=dx, grad_weight=dw, grad_bias=db, accumulate=add)
    assert got is dx and a.intact()
    g, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    d = g * w.double()
    c1, c2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
    want = r * (d - c1 - h * c2)
    tol = r * (6 * U * (d.abs() + c1.abs() + (h * c2).abs()) + _chain(cols) * (d.abs().mean(1, keepdim=True) + h.abs() * (d * h).abs().mean(1, keepdim=True)))
    tol = (tol + HALF[out] * want.abs()) * (1 + HALF[out]) + 1e-40
    assert bool(((dx.double() - want).abs() <= tol).all()), float(((dx.double() - want).abs() / tol).max())
    for got, terms, old in ((dw, g * h, old_w), (db, g, old_b)):
        want = terms.sum(0) + (old if add else 0)
        tol = (rows / 148 + 70) * U * terms.abs().sum(0) + 2 * U * old.abs() + HALF[wdt] * want.abs() * (1 + HALF[wdt]) + 1e-40
        assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() / tol).max())


@pytest.mark.parametrize("rows,cols", [(5000, 256), (3001, 768), (2000, 1001), (700, 4096), (400, 9000)])
def test_backward_of_many_rows_and_twice(env, rows, cols):
    """Sums over many rows; the same call gives the same bits; each output alone is the same as with the others."""
    torch, binding = env
    gen = torch.Generator(device="cuda").manual_seed(9)
    x, dy = (torch.randn(rows, cols, generator=gen, device="cuda") for _ in range(2))
    w = torch.randn(cols, generator=gen, device="cuda")
    _, mean, rstd = binding.layer_norm_forward(x, w)
    run = lambda: [torch.empty(cols, device="cuda") for _ in range(2)]  # noqa: E731
    (dw, db), (dw2, db2) = run(), run()
    dx = binding.layer_norm_backward(dy, x, mean, rstd, w, grad_weight=dw, grad_bias=db)
    dx2 = binding.layer_norm_backward(dy, x, mean, rstd, w, grad_weight=dw2, grad_bias=db2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for got, terms in ((dw, dy.double() * h), (db, dy.double())):
        assert bool(((got.double() - terms.sum(0)).abs() <= (rows / 148 + 70) * U * terms.abs().sum(0)).all())
    assert torch.equal(binding.layer_norm_backward(dy, x, mean, rstd, w), dx)
    (dw3, db3) = run()
    assert binding.layer_norm_backward(dy, x, mean, rstd, w, grad_weight=dw3, need_x=False) is None and torch.equal(dw3, dw)
    binding.layer_norm_backward(dy, x, mean, rstd, w, grad_bias=db3, need_x=False)
    assert torch.equal(db3, db)


def test_gradients_against_differences(env):
    """Central differences of L = sum(y * c) in 64 bits (the formula's own y) with steps of 1e-4: their error is of the order 1e-8 of
    the third derivatives, the kernel's own below 1e-5 of the values here; 1e-4 of the largest gradient holds both."""
    torch, binding = env
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, c = (torch.randn(3, 21, generator=gen, device="cuda") for _ in range(2))
    w, b = (torch.randn(21, generator=gen, device="cuda") for _ in range(2))

    def loss(x, w, b):
        m, v = x.mean(-1, keepdim=True), x.var(-1, unbiased=False, keepdim=True)
        return (((x - m) / (v + 1e-5).sqrt() * w + b) * c.double()).sum()

    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    (binding.layer_norm(*leaves) * c).sum().backward()
    args = [t.double() for t in (x, w, b)]
    for i, leaf in enumerate(leaves):
        diff = torch.empty_like(args[i])
        for k in range(diff.numel()):
            ends = []
            for sign in (1, -1):
                moved = [t.clone() for t in args]
                moved[i].view(-1)[k] += sign * 1e-4
                ends.append(loss(*moved))
            diff.view(-1)[k] = (ends[0] - ends[1]) / 2e-4
        assert float((leaf.grad.double() - diff).abs().max()) <= 1e-4 * float(diff.abs().max())


def test_a_large_common_part_keeps_the_variance(env):
    """Rows around 4096 with deviations of 1: squares' means would cancel to nothing."""
    torch, binding = env
    x = 4096 + torch.randn(64, 4096, device="cuda")
    _, mean, rstd = binding.layer_norm_forward(x)
    want = (x.double().var(1, unbiased=False) + 1e-5) ** -0.5
    # the mean's error e below 42 u 4096 + u 4096 = 1.05e-2: e^2 / 2 of the variance, 6e-5, besides chain
    assert bool(((rstd.double() - want).abs() <= want * 7e-5).all())


def test_constant_rows_infinities_and_nan(env):
    torch, binding = env
    x = torch.randn(6, 300, device="cuda")
    x[1] = 2.5
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    y, mean, rstd = binding.layer_norm_forward(x, eps=0.0)
    assert y[1].isnan().all() and bool(rstd[1].isinf())               # 0 / sqrt(0), as the formula gives it
    assert y[2].isnan().all() and y[3].isnan().all()
    assert y[[0, 4, 5]].isfinite().all()
    y, mean, rstd = binding.layer_norm_forward(x, eps=1e-6)
    assert bool((y[1] == 0).all()) and abs(float(rstd[1]) - 1e3) < 1e-2
    dw = torch.empty(300, device="cuda")
    dx = binding.layer_norm_backward(torch.ones_like(x), x, mean, rstd, torch.ones(300, device="cuda"), grad_weight=dw)
    assert dx[2].isnan().all() and dx[[0, 1, 4, 5]].isfinite().all() and dw.isnan().all()


def test_no_rows(env):
    torch, binding = env
    x = torch.empty(0, 64, device="cuda")
    y, mean, rstd = binding.layer_norm_forward(x)
    assert y.shape == x.shape and mean.shape == (0,)
    dw, db = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    binding.layer_norm_backward(x, x, mean, rstd, None, grad_weight=dw, grad_bias=db, accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    binding.layer_norm_backward(x, x, mean, rstd, None, grad_weight=dw, grad_bias=db)
    assert not dw.any() and not db.any()


def test_shapes_strides_and_autograd(env):
    torch, binding = env
    x = torch.randn(4, 6, 5, 128, device="cuda", requires_grad=True)
    w, b = torch.randn(64, device="cuda", requires_grad=True), torch.randn(64, device="cuda", requires_grad=True)
    y = binding.layer_norm(x[..., :64], w, b)                          # rows at one stride
    y.sum().backward()
    first = [t.grad.clone() for t in (x, w, b)]
    for t in (x, w, b):
        t.grad = None
    torch.nn.functional.layer_norm(x[..., :64], (64,), w, b).sum().backward()
    for t, f in zip((x, w, b), first):                                 # two fp32 computations of sums of up to 64 terms near 1
        assert torch.allclose(f, t.grad, rtol=0, atol=2e-5)
    with torch.no_grad():
        assert not binding.layer_norm(x[..., 64:], w, b).requires_grad
    frozen = binding.layer_norm(x.detach()[..., 64:], w.detach(), b)
    frozen.sum().backward()
    with pytest.raises(binding.CameError) as e:
        binding.layer_norm_forward(x.detach()[:, :, 1:3])               # two strides
    assert e.value.status == 11


def test_captured_and_on_another_stream(env):
    torch, binding = env
    x, w = torch.randn(500, 768, device="cuda"), torch.randn(768, device="cuda")
    dw, db = torch.zeros(768, device="cuda"), torch.zeros(768, device="cuda")

    def work():
        y, mean, rstd = binding.layer_norm_forward(x, w)
        return y, binding.layer_norm_backward(y, x, mean, rstd, w, grad_weight=dw, grad_bias=db, accumulate=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for k in range(3):
        x.normal_()
        dw.zero_(); db.zero_()
        graph.replay()
        got_sums = dw.clone(), db.clone()
        dw.zero_(); db.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = work()
        side.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(got_sums[0], dw) and torch.equal(got_sums[1], db)


def test_more_than_two_to_the_31_elements(env):
    """Rows behind the 2^31st element of x and y."""
    torch, binding = env
    rows, cols = 262_200, 8192
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, cols, device="cuda").bfloat16()
    y, mean, rstd = binding.layer_norm_forward(x)
    assert not y[:-3].any()
    _check_forward(torch, x[-3:], None, None, 1e-5, y[-3:], mean[-3:], rstd[-3:], "bf16")
    dy = torch.zeros_like(x)
    dy[-3:] = torch.randn(3, cols, device="cuda").bfloat16()
    dw = torch.empty(cols, device="cuda")
    binding.layer_norm_backward(dy, x, mean, rstd, None, grad_x=y, grad_weight=dw)
    h = (x[-3:].double() - mean[-3:].double()[:, None]) * rstd[-3:].double()[:, None]
    terms = dy[-3:].double() * h
    assert bool(((dw.double() - terms.sum(0)).abs() <= 10 * U * terms.abs().sum(0)).all())
    assert not y[:-3].any() and y[-3:].any()


def test_refusals(env):
    torch, binding = env
    x, w = torch.randn(4, 64, device="cuda"), torch.randn(64, device="cuda")
    f, g = binding.layer_norm_forward, binding.layer_norm_backward
    m = torch.zeros(4, device="cuda")
    for bad, status in (
            (lambda: f(x.cpu()), 7), (lambda: f(x.half()), 3), (lambda: f(x, w[:5]), 2), (lambda: f(x, w.cpu()), 7), (lambda: f(x, w, w.bfloat16()), 3),
            (lambda: f(x[:, ::2]), 11), (lambda: f(x, out=x), 12), (lambda: f(x, out=x.new_empty(4, 63)), 2), (lambda: f(x, eps=-1.0), 5),
            (lambda: f(torch.zeros((), device="cuda")), 2), (lambda: f(x, out_dtype=torch.float16), 3), (lambda: f(x, w[::2].repeat(2)[::1], w.view(1, 64)), 2),
            (lambda: g(x, x[:3], m[:3], m[:3]), 2), (lambda: g(x, x, m[:3], m), 2), (lambda: g(x, x, m.double(), m), 3), (lambda: g(x, x, m, m, w, grad_weight=w), 12),
            (lambda: g(x, x, m, m, w, grad_weight=w.bfloat16()), 3), (lambda: g(x, x, m, m, w, grad_x=x), 12), (lambda: g(x, x, m.cpu(), m), 7)):
        with pytest.raises(binding.CameError) as e:
            bad()
        assert e.value.status == status, e.value


@pytest.mark.parametrize("rows,cols,extra,offset", [(70001, 64, 0, 0), (20001, 250, 0, 0), (16385, 256, 8, 0), (9001, 513, 0, 1), (5001, 1000, 0, 0), (3003, 2050, 2, 0),
                                                    (1031, 4096, 0, 0), (901, 5120, 0, 0), (515, 8192, 0, 8), (300, 16384, 0, 0), (297, 12296, 0, 0)])
@pytest.mark.parametrize("dtype,out,wdt", [("f32", "f32", "bf16"), ("bf16", "bf16", "f32")])
def test_many_rows_in_both_directions(env, rows, cols, extra, offset, dtype, out, wdt):
    """Groups that go from row to row, with full and partly filled last turns."""
    torch, binding = env
    a = Arena(torch)
    x, w, b, new = _inputs(torch, a, rows, cols, cols + extra, offset, dtype, wdt, 15)
    y = a.matrix(rows, cols, cols + extra, offset, out)
    _, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-5, out=y)
    _check_forward(torch, x, w, b, 1e-5, y, mean, rstd, out)
    dy, dx = a.matrix(rows, cols, cols + extra, offset, dtype), a.matrix(rows, cols, cols + extra, offset, dtype)
    dy.copy_(new(rows, cols))
    dw, db = torch.empty_like(w), torch.empty_like(w)
    binding.layer_norm_backward(dy, x, mean, rstd, w, grad_x=dx, grad_weight=dw, grad_bias=db)
    assert a.intact()
    g, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    d = g * w.double()
    c1, c2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
    want = r * (d - c1 - h * c2)
    tol = r * (6 * U * (d.abs() + c1.abs() + (h * c2).abs()) + _chain(cols) * (d.abs().mean(1, keepdim=True) + h.abs() * (d * h).abs().mean(1, keepdim=True)))
    tol = (tol + HALF[dtype] * want.abs()) * (1 + HALF[dtype]) + 1e-40
    assert bool(((dx.double() - want).abs() <= tol).all())
    for got, terms in ((dw, g * h), (db, g)):
        tol = (rows / 148 + 70) * U * terms.abs().sum(0) + HALF[wdt] * terms.sum(0).abs() * (1 + HALF[wdt]) + 1e-40
        assert bool(((got.double() - terms.sum(0)).abs() <= tol).all())


@pytest.mark.parametrize("cols", [1001, 1002, 1004, 771, 100, 5003, 9001])
@pytest.mark.parametrize("dtype,mixed", [("f32", False), ("bf16", False), ("bf16", True)])
def test_contiguous_rows_of_odd_lengths(env, cols, dtype, mixed):
    """Rows that begin at other places relative to an aligned address; whatever a tensor's neighbours in memory hold stays out of it."""
    torch, binding = env
    rows = 5 + (5 << 20) // cols
    gen = torch.Generator(device="cuda").manual_seed(cols)
    dt, gdt = _dt(torch, dtype), torch.float32 if mixed else _dt(torch, dtype)

    def between(dt):                     # a tensor between NaN, starting at an aligned address
        flat = torch.full((64 + rows * cols + 64,), float("nan"), dtype=dt, device="cuda")
        view = flat[64:64 + rows * cols].view(rows, cols)
        return flat, view
    (fx, x), (fy, y), (fg, dy), (fd, dx) = between(dt), between(gdt), between(gdt), between(dt)
    x.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    x[3], x[4, 0], x[0, -1] = float("inf"), float("nan"), float("inf")       # neighbours of rows 2, 3, 5 and 1
    dy.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
    w, b = torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    _, mean, rstd = binding.layer_norm_forward(x, w, b, out=y)
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[[0, 3, 4]] = False
    assert bool(y[good].isfinite().all()) and bool(y[~good].isnan().any(1).all())
    _check_forward(torch, x[good], w, b, 1e-5, y[good], mean[good], rstd[good], "f32" if gdt == torch.float32 else "bf16")
    binding.layer_norm_backward(dy, x, mean, rstd, w, grad_x=dx)
    assert bool(dx[good].isfinite().all())
    x[~good] = 1.0
    _, mean, rstd = binding.layer_norm_forward(x, w, b, out=y)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    binding.layer_norm_backward(dy, x, mean, rstd, w, grad_x=dx, grad_weight=dw, grad_bias=db)
    for flat in (fx, fy, fg, fd):
        assert bool(flat[:64].isnan().all()) and bool(flat[-64:].isnan().all())
    g, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    d = g * w.double()
    c1, c2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
    want = r * (d - c1 - h * c2)
    tol = r * (6 * U * (d.abs() + c1.abs() + (h * c2).abs()) + _chain(cols) * (d.abs().mean(1, keepdim=True) + h.abs() * (d * h).abs().mean(1, keepdim=True)))
    tol = (tol + HALF[dtype] * want.abs()) * (1 + HALF[dtype]) + 1e-40
    assert bool(((dx.double() - want).abs() <= tol).all())
    for got, terms in ((dw, g * h), (db, g)):
        assert bool(((got.double() - terms.sum(0)).abs() <= (rows / 148 + 70) * U * terms.abs().sum(0) + 1e-40).all())


def test_sums_over_many_long_rows(env):
    """Rows beyond a block, 9000 of them and all of one sign: a warp adds 512 at most one after another."""
    torch, binding = env
    rows, cols = 9000, 20000
    x = torch.randn(rows, cols, device="cuda").bfloat16()
    dy = torch.rand(rows, cols, device="cuda").bfloat16()
    _, mean, rstd = binding.layer_norm_forward(x)
    db = torch.empty(cols, device="cuda")
    binding.layer_norm_backward(dy, x, mean, rstd, grad_bias=db, need_x=False)
    want = sum(part.double().sum(0) for part in dy.split(1000))
    assert bool(((db.double() - want).abs() <= (512 + 40) * U * want).all())


def test_sums_over_a_very_long_row(env):
    """2^27 - 1 equal numbers, whose roundings all go one way: a thread adds 256 in a row, then at most 512 such sums, and 10 levels
    across the block; the mean's own factor and product are two more."""
    torch, binding = env
    x = torch.full((1, (1 << 27) - 1), 0.1, device="cuda")
    value = float(x[0, 0])
    e = (256 + 512 + 12) * U * value
    y, mean, rstd = binding.layer_norm_forward(x)
    assert abs(float(mean) - value) <= e
    assert float(y.abs().max()) <= 2 * e * 1e-5 ** -0.5                  # the mean's error, and the differences' rounding
    # the variance: squares of 0.1 (every second element has the other sign: the mean is 0.1 / n)
    x[0, 1::2] = -value
    _, _, rstd = binding.layer_norm_forward(x)
    want = (value ** 2 + 1e-5) ** -0.5
    assert abs(float(rstd) - want) <= want * ((256 + 512 + 16) * U / 2 + 3 * U)
    # d is the same everywhere, and its mean is taken off: nothing is left but the mean's error
    dx = binding.layer_norm_backward(torch.full_like(x, value), x, torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"))
    assert float(dx.abs().max()) <= 2 * e
