"""The relative position bias bit for bit, and its gradient against the formula in 64 bits.

A sum of N terms is formed in fp32: a diagonal's in one register, a term for each eighth row of a part of at most 128 such rows and for
each batch of a warp, then at most 8 diagonals of a lane one after another and 5 levels across the warp (a short interval: 32 diagonals),
units / 32 + 32 at the end.  For the sizes here (at most 3 batches, 1024 units) a term passes at most 3 * 128 + 32 + 64 additions,
and no more than 512: the error is below 512 u of the sum of magnitudes (u = 2^-24), plus half a step of the stored type."""
import numpy as np
import pytest

from tests.test_posbias_cpu import bucket

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _dt(torch, name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _buckets(torch, q, k, offset, n, far, both):
    line = torch.tensor([bucket(r - offset, n, far, both) for r in range(1 - q, k)], dtype=torch.int64, device="cuda")
    return line[torch.arange(k, device="cuda")[None] - torch.arange(q, device="cuda")[:, None] + q - 1]


CASES = [
    # heads, q, k, offset, buckets, far, both
    (1, 1, 1, 0, 32, 128, True), (3, 1, 2048, 2047, 32, 128, False), (2, 1, 777, 100, 32, 128, True), (5, 7, 3, 0, 8, 20, True), (2, 9, 8, -4, 4, 3, True),
    (2, 63, 65, 2, 32, 128, False), (1, 300, 1, 299, 32, 128, False), (12, 128, 128, 0, 32, 128, True), (2, 257, 1025, 700, 32, 128, True),
    (3, 513, 264, 0, 64, 1000, False), (1, 1000, 2050, 1050, 32, 128, False), (2, 130, 1032, 1 << 39, 32, 128, False), (2, 130, 1032, -(1 << 39), 32, 128, True),
    (1, 700, 3, 0, 1024, 5000, True), (2, 96, 4099, 0, 2, 2, False), (40, 33, 47, 14, 32, 40, True),
]


@pytest.mark.parametrize("heads,q,k,offset,n,far,both", CASES)
@pytest.mark.parametrize("tdt,out", [("f32", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")])
def test_forward(env, heads, q, k, offset, n, far, both, tdt, out):
    torch, binding = env
    wide = torch.randn(n, heads + 3, device="cuda").to(_dt(torch, tdt))
    table = wide[:, 1:heads + 1]
    want = table.float()[_buckets(torch, q, k, offset, n, far, both)].permute(2, 0, 1).to(_dt(torch, out))
    for shift in (0, 1, 5):              # other alignments of the first row, guards on both sides
        arena = torch.full((64 + shift + heads * q * k + 64,), -7.25, dtype=_dt(torch, out), device="cuda")
        view = arena[64 + shift:64 + shift + heads * q * k].view(heads, q, k)
        got = binding.position_bias_forward(table, q, k, offset, both, far, out=view)
        assert got is view and torch.equal(view, want)
        assert bool((arena[:64 + shift] == -7.25).all()) and bool((arena[64 + shift + heads * q * k:] == -7.25).all())
    if abs(offset) < 1 << 31:
        on_device = torch.tensor(offset, device="cuda")
        assert torch.equal(binding.position_bias_forward(table, q, k, on_device, both, far, out_dtype=_dt(torch, out)), want)


@pytest.mark.parametrize("heads,q,k,offset,n,far,both", CASES)
@pytest.mark.parametrize("batch,dt,tdt,add", [(1, "f32", "f32", False), (3, "bf16", "f32", True), (2, "bf16", "bf16", False), (1, "f32", "bf16", True)])
def test_backward(env, heads, q, k, offset, n, far, both, batch, dt, tdt, add):
    torch, binding = env
    gen = torch.Generator(device="cuda").manual_seed(7)
    dout = torch.randn(batch, heads, q, k, generator=gen, device="cuda").to(_dt(torch, dt))
    wide = torch.randn(n, heads + 3, generator=gen, device="cuda").to(_dt(torch, tdt))
    before, grad = wide.clone(), wide[:, 1:heads + 1]
    old = grad.double()
    assert binding.position_bias_backward(dout, grad, offset, both, far, accumulate=add) is grad
    where = _buckets(torch, q, k, offset, n, far, both).view(-1)
    sums, sizes = (torch.zeros(n, heads, dtype=torch.float64, device="cuda").index_add_(0, where, x.sum(0).view(heads, -1).t()) for x in (dout.double(), dout.double().abs()))
    want = sums + (old if add else 0)
    tol = 512 * U * sizes + U * old.abs() + HALF[tdt] * want.abs() * (1 + HALF[tdt]) + 1e-40
    assert bool(((grad.double() - want).abs() <= tol).all()), float(((grad.double() - want).abs() / tol).max())
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, heads + 1:], before[:, heads + 1:])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_strides_and_broadcasts_of_the_gradient(env, dt):
    """Slices, transposed heads, odd offsets and broadcast (stride 0) dimensions give what a contiguous copy gives."""
    torch, binding = env
    base = torch.randn(2, 70, 5, 300, device="cuda").to(_dt(torch, dt))            # (batch, query, head, key)
    for view in (base.transpose(1, 2), base[:, 3:60, :, 1:288].transpose(1, 2), base[:, ::2, 1:, 16:272].transpose(1, 2), base[0].transpose(0, 1),
                 base[:, :1].transpose(1, 2).expand(-1, -1, 33, -1), base[:1, :, :1].transpose(1, 2).expand(3, 4, -1, -1)):
        heads = view.shape[-3]
        got, want = (binding.position_bias_backward(x, torch.empty(32, heads, device="cuda"), 5) for x in (view, view.contiguous()))
        # the same terms, perhaps in tiles of another alignment
        sizes = binding.position_bias_backward(view.abs().contiguous(), torch.empty(32, heads, device="cuda"), 5)
        assert bool(((got - want).abs() <= 2 * 512 * U * sizes).all())
        assert torch.equal(got, binding.position_bias_backward(view, torch.empty(32, heads, device="cuda"), 5))      # bit for bit


def test_gradient_against_differences(env):
    """The bias is linear in the table: its gradient in whole numbers is exact, and equals the change of the sum for a change of one."""
    torch, binding = env
    table = torch.randint(-4, 5, (8, 3), device="cuda").float().requires_grad_()
    weight = torch.randint(-3, 4, (3, 20, 31), device="cuda").float()
    (binding.position_bias_forward(table, 20, 31, 2, True, 12) * weight).sum().backward()
    with torch.no_grad():
        base = (binding.position_bias_forward(table, 20, 31, 2, True, 12) * weight).sum()
        for b in range(8):
            for h in range(3):
                moved = table.clone()
                moved[b, h] += 1
                assert float((binding.position_bias_forward(moved, 20, 31, 2, True, 12) * weight).sum() - base) == float(table.grad[b, h])


def test_autograd_with_a_batch_and_an_expanded_gradient(env):
    torch, binding = env
    table = torch.randn(32, 4, device="cuda", requires_grad=True)
    scores = torch.randn(3, 4, 40, 50, device="cuda")
    (scores + binding.position_bias_forward(table, 40, 50)).sum().backward()           # an expanded gradient reaches the bias
    where = _buckets(torch, 40, 50, 0, 32, 128, True).view(-1)
    want = torch.bincount(where, minlength=32).float() * 3
    assert torch.equal(table.grad, want[:, None].expand(-1, 4))
    with pytest.raises(binding.CameError) as e:
        binding.position_bias_forward(table, 4, 5, out=torch.empty(4, 4, 5, device="cuda"))
    assert e.value.status == 11


def test_captured_decoding_counts_on_the_device(env):
    torch, binding = env
    table = torch.randn(32, 12, device="cuda")
    t = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        row = binding.position_bias_forward(table, 1, 2048, t, bidirectional=False)
        t += 1
    for k in range(4):
        t.fill_(500 * k)
        graph.replay()
        assert torch.equal(row, binding.position_bias_forward(table, 1, 2048, 500 * k, bidirectional=False)) and int(t) == 500 * k + 1


def test_infinities_reach_their_bucket_alone(env):
    torch, binding = env
    dout = torch.ones(1, 64, 64, device="cuda")
    dout[0, 10, 15] = float("inf")
    dout[0, 20, 17] = float("nan")
    grad = binding.position_bias_backward(dout, torch.empty(32, 1, device="cuda"))
    bad = ~grad[:, 0].isfinite()
    assert bad.sum() == 2 and grad[bucket(5, 32, 128, True), 0].isinf() and grad[bucket(-3, 32, 128, True), 0].isnan()


def test_empty(env):
    torch, binding = env
    table = torch.randn(32, 4, device="cuda")
    assert binding.position_bias_forward(table, 0, 5).shape == (4, 0, 5) and binding.position_bias_forward(table, 5, 0).shape == (4, 5, 0)
    for shape in ((4, 0, 5), (4, 5, 0), (0, 4, 5, 5)):
        grad = torch.ones(32, 4, device="cuda")
        binding.position_bias_backward(torch.empty(shape, device="cuda"), grad, accumulate=True)
        assert bool((grad == 1).all())
        binding.position_bias_backward(torch.empty(shape, device="cuda"), grad)
        assert not grad.any()


def test_more_than_two_to_the_31_elements(env):
    torch, binding = env
    heads, q, k = 9, 16384, 16392
    table = torch.randn(32, heads, device="cuda")
    out = binding.position_bias_forward(table, q, k, out_dtype=torch.bfloat16)
    assert out.numel() > 1 << 31
    for h, i in ((0, 0), (8, q - 1), (8, 5000)):
        want = table[:, h][torch.tensor([bucket(j - i, 32, 128, True) for j in range(k)], device="cuda")].bfloat16()
        assert torch.equal(out[h, i], want)
    out.zero_()
    out[8, -1, -1] = 2.0
    out[8, 5000, 4990] = 3.0
    grad = binding.position_bias_backward(out, torch.empty(32, heads, device="cuda"))
    assert float(grad[bucket(k - q, 32, 128, True), 8]) == 2.0 and float(grad[bucket(-10, 32, 128, True), 8]) == 3.0 and int((grad != 0).sum()) == 2


def test_refusals(env):
    torch, binding = env
    t = torch.randn(32, 4, device="cuda")
    f, g = binding.position_bias_forward, binding.position_bias_backward
    d = torch.randn(4, 5, 6, device="cuda")
    for bad, status in (
            (lambda: f(t.cpu(), 3, 3), 7), (lambda: f(t.half(), 3, 3), 3), (lambda: f(t[0], 3, 3), 2), (lambda: f(t, -1, 3), 2), (lambda: f(t, 3, 3, max_distance=8), 5),
            (lambda: f(t[:31], 3, 3), 2), (lambda: f(t, 3, 3, offset=0.5), 3), (lambda: f(t, 3, 3, offset=torch.zeros(1, device="cuda")), 3),
            (lambda: f(t, 3, 3, offset=torch.zeros(1, dtype=torch.int64)), 7), (lambda: f(t, 3, 3, out=torch.empty(4, 3, 4, device="cuda")), 2),
            (lambda: f(t, 3, 3, out=torch.empty(4, 3, 6, device="cuda")[:, :, ::2]), 11), (lambda: f(t, 3, 3, out_dtype=torch.float16), 3),
            (lambda: f(t.t(), 3, 3), 11), (lambda: g(d[:3], t), 2), (lambda: g(d[0], t), 2), (lambda: g(d.half(), t), 3), (lambda: g(d.cpu(), t), 7),
            (lambda: g(d.transpose(1, 2), t), 11), (lambda: g(d, t, bidirectional=False, max_distance=16), 5)):
        with pytest.raises(binding.CameError) as e:
            bad()
        assert e.value.status == status, e.value


@pytest.mark.parametrize("dt,heads,q,k,batch,expanded", [("f32", 64, 64, 64, 65536, True), ("f32", 64, 512, 520, 300, True), ("f32", 12, 333, 517, 257, True),
                                                         ("f32", 1, 100, 90, 40000, True), ("f32", 1, 99, 91, 40001, False), ("bf16", 2, 63, 200, 3000, False)])
def test_large_batches_of_one_sign(env, dt, heads, q, k, batch, expanded):
    """Sums of equal numbers, whose roundings all go one way: at most 512 additions in a row for a lane's diagonal, 32 for the diagonals
    of a bucket, 16 for the warps' sums, then 64 bits, and the rounding at the end: 561 u of the sum."""
    torch, binding = env
    one = torch.full((1, heads, q, k), 0.1, device="cuda").to(_dt(torch, dt))
    dout = one.expand(batch, -1, -1, -1) if expanded else one.repeat(batch, 1, 1, 1)
    grad = binding.position_bias_backward(dout, torch.empty(32, heads, device="cuda"))
    count = torch.bincount(_buckets(torch, q, k, 0, 32, 128, True).view(-1), minlength=32).double()
    want = (count * batch * float(one[0, 0, 0, 0]))[:, None].expand(-1, heads)
    assert bool(((grad.double() - want).abs() <= 561 * U * want).all()), float(((grad.double() - want).abs() / want.clamp(min=1e-9)).max()) / U


def test_numbers_beyond_the_descriptor_are_refused(env):
    """Offsets beyond 64 bits, distances beyond 32 and lengths beyond the limits: as the library refuses smaller ones, before anything is allocated."""
    torch, binding = env
    t, d = torch.randn(32, 4, device="cuda"), torch.randn(4, 5, 6, device="cuda")
    f, g = binding.position_bias_forward, binding.position_bias_backward
    for bad, status in (
            (lambda: f(t, 3, 3, offset=1 << 64), 2), (lambda: f(t, 3, 3, offset=-(1 << 40) - 1), 2), (lambda: f(t, 3, 3, max_distance=1 << 33), 5),
            (lambda: f(t, 3, 3, max_distance=-(1 << 40)), 5), (lambda: f(t, 3, 3, max_distance=128.0), 5), (lambda: f(t, 1 << 40, 1), 2), (lambda: f(t, 1, 1 << 70), 2),
            (lambda: g(d, t, offset=1 << 64), 2), (lambda: g(d, t, offset=(1 << 40) + 1), 2), (lambda: g(d, t, max_distance=1 << 33), 5),
            (lambda: f(t.clone().requires_grad_(), 3, 3, offset=1 << 64), 2), (lambda: f(t.clone().requires_grad_(), 3, 3, max_distance=1 << 33), 5)):
        with pytest.raises(binding.CameError) as e:
            bad()
        assert e.value.status == status, e.value
    assert torch.equal(f(t, 2, 3, offset=1 << 40), f(t, 2, 3, offset=1 << 20)) and torch.equal(f(t, 2, 3, max_distance=np.int64(99)), f(t, 2, 3, max_distance=99))
