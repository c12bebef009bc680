"""The AdamW step against its formulas: states and codes bit for bit, parameters in 64 bits."""
import numpy as np
import pytest

from tests import adamw_reference as ref

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
SENT = 77


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _guarded(torch, n, dtype, offset):
    """A view of n zeros, `offset` elements after a 256-byte boundary, and its guards' check."""
    size = torch.empty(0, dtype=dtype).element_size()
    arena = torch.full((256 + (offset + n) * size + 256,), SENT, dtype=torch.uint8, device="cuda")
    a, b = 256 + offset * size, 256 + (offset + n) * size
    arena[a:b] = 0
    return arena[a:b].view(dtype), lambda: bool((arena[:a] == SENT).all()) and bool((arena[b:] == SENT).all())


class Pair:
    """An optimizer over guarded tensors beside the reference."""

    def __init__(self, env, sizes, offsets, gdt, bits, copy=False, flags=None, seed=3, spread=1.0, start=0):
        torch, self.binding = env
        self.torch, self.sizes, self.seed, self.flags = torch, sizes, seed, flags or [0] * len(sizes)
        self.bits = [bits] * len(sizes) if isinstance(bits, int) else bits
        self.guards, self.t = [], start
        new = lambda n, dt, off: self._keep(_guarded(torch, n, dt, off))  # noqa: E731
        rng = np.random.default_rng(seed)
        gdts = [gdt] * len(sizes) if isinstance(gdt, str) else gdt
        gd = [torch.float32 if x == "f32" else torch.bfloat16 for x in gdts]
        self.p = [new(n, torch.float32, o) for n, o in zip(sizes, offsets)]
        self.g = [new(n, d, o) for n, o, d in zip(sizes, offsets, gd)]
        for p in self.p:
            p.copy_(torch.from_numpy(rng.normal(0, 0.02, p.numel()).astype(np.float32)))
        st = lambda k: [new(n, (torch.float32 if b == 32 else k), o) for n, o, b in zip(sizes, offsets, self.bits)]  # noqa: E731
        sc = lambda: [new(-(-n // 256), torch.uint8, o).view(torch.float8_e8m0fnu) if b == 8 else None for n, o, b in zip(sizes, offsets, self.bits)]  # noqa: E731
        self.m, self.v, self.ms, self.vs = st(torch.float8_e4m3fn), st(torch.float8_e5m2), sc(), sc()
        self.copy = [new(n, torch.bfloat16, o) for n, o in zip(sizes, offsets)] if copy else None
        self.rng, self.spread = rng, spread
        self.opt = self.binding.AdamWOptimizer(self.p, self.g, state_bits=self.bits, flags=self.flags, m=self.m, v=self.v, m_scale=self.ms,
                                               v_scale=self.vs, bf16_copy=self.copy if copy else False, seed=seed, step_count=start)

    def _keep(self, pair):
        self.guards.append(pair[1])
        return pair[0]

    def new_gradients(self):
        for i, g in enumerate(self.g):
            x = self.rng.normal(0, self.spread * 10.0 ** -(i % 4), g.numel()) * np.exp(self.rng.normal(0, 2, g.numel()))
            g.copy_(self.torch.from_numpy(x.astype(np.float32)))

    def bytes_of(self, x):
        return x.view(self.torch.uint8).cpu().numpy()

    def check_step(self, hp=HP, scale=1.0, **kw):
        before = [self.read(i) for i in range(len(self.sizes))]
        self.opt.step(**hp, **kw)
        self.t += 1
        block0 = 0
        for i, n in enumerate(self.sizes):
            p, g, m, v, *_ = before[i]
            want_p, m, v, tol = ref.step(p, g, m, v, hp, self.t, scale, not self.flags[i])
            p2, _, m2, v2, cm, cv, sm, sv = self.read(i)
            if self.bits[i] == 32:
                np.testing.assert_array_equal(m2, m)
                np.testing.assert_array_equal(v2, v)
            else:
                r = ref.random_bits(n, block0, self.seed, self.t)
                em, es = ref.encode(m, r & np.uint64(0xFFFF), ref.E4M3, 7, True)
                np.testing.assert_array_equal(sm, es)
                np.testing.assert_array_equal(np.where(cm & 127 == 127, 127, cm), em)       # (a NaN's sign says nothing)
                ev, es = ref.encode(v, r >> np.uint64(16), ref.E5M2, 14, False)
                np.testing.assert_array_equal(sv, es)
                np.testing.assert_array_equal(cv, ev)
            fine = np.isfinite(want_p)
            assert np.array_equal(fine, np.isfinite(p2))
            assert (np.abs(p2[fine] - want_p[fine]) <= tol[fine]).all(), np.max(np.abs(p2[fine] - want_p[fine]) / tol[fine])
            if self.copy:
                assert self.torch.equal(self.copy[i].view(self.torch.int16), self.p[i].to(self.torch.bfloat16).view(self.torch.int16))
            block0 += -(-n // 256)
        assert all(ok() for ok in self.guards)

    def read(self, i):
        p, g = self.p[i].cpu().numpy(), self.g[i].float().cpu().numpy()
        if self.bits[i] == 32:
            return p, g, self.m[i].cpu().numpy(), self.v[i].cpu().numpy(), None, None, None, None
        cm, cv, sm, sv = (self.bytes_of(x[i]) for x in (self.m, self.v, self.ms, self.vs))
        return p, g, ref.decode(cm, sm, ref.E4M3, True), ref.decode(cv, sv, ref.E5M2, False), cm, cv, sm, sv


LISTS = [
    ([1], [0]), ([0, 5, 0], [0, 3, 0]), ([7, 8, 9, 31, 32, 33], [0, 1, 2, 3, 4, 5]), ([255, 256, 257, 511, 512, 513], [0, 0, 0, 8, 1, 0]),
    ([2048, 2049, 4095, 8192 + 7], [0, 0, 1, 0]), ([65 * 33, 1, 7, 300, 70001], [0, 3, 1, 0, 16]), ([3] * 700, [0] * 700),
]


@pytest.mark.parametrize("k", range(len(LISTS)))
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt,copy", [("f32", False), ("bf16", True)])
def test_steps_against_the_formulas(env, gdt, copy, bits, k):
    sizes, offsets = LISTS[k]
    pair = Pair(env, sizes, offsets, gdt, bits, copy, flags=[i % 2 for i in range(len(sizes))])
    for _ in range(3):
        pair.new_gradients()
        pair.check_step()


def test_mixed_list(env):
    n = 6
    pair = Pair(env, [300, 1000, 256, 5000, 77, 4096], [0] * n, ["f32", "bf16", "f32", "bf16", "bf16", "f32"], [8, 32, 32, 8, 8, 32])
    for _ in range(2):
        pair.new_gradients()
        pair.check_step()


@pytest.mark.parametrize("bits", [32, 8])
def test_hyper_parameters_scales_and_late_steps(env, bits):
    torch, _ = env
    pair = Pair(env, [1000, 513], [0, 0], "f32", bits, start=123456)
    coef = torch.tensor([0.37], device="cuda")
    for hp in (HP, dict(lr=0.0, beta1=0.0, beta2=0.0, eps=1e-3), dict(lr=1e-3, beta1=0.95, beta2=0.95, eps=1e-6, weight_decay=0.0),
               dict(lr=1e-3, beta1=0.5, beta2=0.99999, eps=0.0, weight_decay=1.0)):
        pair.new_gradients()
        pair.check_step(hp)
        pair.check_step(hp, scale=np.float32(0.25) * coef.cpu().numpy()[0], grad_scale=0.25, device_scale=coef)


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_values_at_the_ends_of_the_range(env, gdt):
    """Zeros, subnormal and huge values, infinities and NaN in some elements of a block: the others are stored as ever."""
    pair = Pair(env, [1024, 300], [0, 0], gdt, 8)
    # (the square of 1e30 overflows: v becomes infinite without an infinity in the gradient)
    odd = np.array([0.0, -0.0, 1e-45, -1e-40, 1e-30, 1e18, -1e18, 1e30, np.inf, -np.inf, np.nan], dtype=np.float32)
    for turn in range(3):
        pair.new_gradients()
        for g in pair.g:
            g[5:16].copy_(pair.torch.from_numpy(odd).to(g.dtype))
            g[280:291].copy_(pair.torch.from_numpy(odd[::-1].copy()).to(g.dtype))
        pair.g[0][512:768] = 0.0
        pair.g[0][768:] = 1e-41
        pair.check_step()


def test_blocks_of_zeros_stay_zero(env):
    torch, binding = env
    p, g = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    opt = binding.AdamWOptimizer([p], [g], state_bits=8)
    opt.step(lr=0.1)
    assert bool((p == 1).all()) and not opt.m[0].float().any() and not opt.v[0].float().any()


def test_same_seed_same_bits_other_seed_other_bits(env):
    torch, binding = env
    g = torch.randn(100_000, device="cuda")

    def run(seed):
        p = torch.zeros_like(g)
        opt = binding.AdamWOptimizer([p], [g], state_bits=8, seed=seed)
        for _ in range(3):
            opt.step(lr=1e-3)
        return p, opt.m[0].view(torch.uint8).clone(), opt.v[0].view(torch.uint8).clone()
    a, b, c = run(1), run(1), run((1 << 63) + 5)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert 0.1 < float((a[1] != c[1]).float().mean()) and 0.1 < float((a[2] != c[2]).float().mean())


def test_mean_of_eight_bit_states_is_the_moving_average(env):
    """With a constant gradient of 1, 300 steps.  One rounding at a time is unbiased (its probabilities are
    centred to 2^-17 of a spacing, v's drift is 2^-8 of one), so the mean over N elements differs from the exact
    average by chance alone: a step's variance is at most spacing x drift, drifts add up to the value itself, so
    a value's variance stays below spacing x value <= value^2 / 4 and the mean's deviation below value / (2 sqrt N); six of them
    for N = 2^18."""
    torch, binding = env
    n, steps = 1 << 18, 300
    p, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    opt = binding.AdamWOptimizer([p], [g], state_bits=8, seed=11)
    for _ in range(steps):
        opt.step(lr=0.0)
    scale = lambda s: torch.exp2(s.view(torch.uint8).double() - 127).repeat_interleave(256)  # noqa: E731
    m, v = (opt.m[0].double() * scale(opt.m_scale[0])).mean(), (opt.v[0].double() * scale(opt.v_scale[0])).mean()
    for got, beta in ((m, 0.9), (v, 0.999)):
        want = 1 - beta ** steps
        assert abs(float(got) - want) <= want * (3 / n ** 0.5 + 2.0 ** -8), (float(got), want)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_on_the_device(env, bits):
    torch, binding = env
    grads = [torch.randn(n, device="cuda") for n in (70_000, 33, 256)]

    def fresh():
        ps = [torch.linspace(-1, 1, g.numel(), device="cuda") for g in grads]
        return ps, binding.AdamWOptimizer(ps, grads, state_bits=bits, seed=5)
    eager_p, eager = fresh()
    graph_p, opt = fresh()
    t, coef = torch.zeros((), dtype=torch.int64, device="cuda"), torch.ones((), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step(lr=0.0, device_step=t, device_scale=coef * 0.0)     # warm-up outside the capture: states stay zero
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t += 1
        opt.step(lr=1e-2, weight_decay=0.1, device_step=t, device_scale=coef)
    assert opt.step_count == 0
    for k in range(1, 6):
        coef.fill_(1.0 / k)
        graph.replay()
        eager.step(lr=1e-2, weight_decay=0.1, device_scale=coef)
        assert int(t) == k
    raw = lambda x: x.view(torch.uint8)  # noqa: E731
    for a, b in zip(eager.m + eager.v, opt.m + opt.v):
        assert torch.equal(raw(a), raw(b))
    for a, b in zip(eager_p, graph_p):       # the device's and the host's expm1 may round a factor differently: 2^-23 of five updates
        assert bool(((a - b).abs() <= 5 * 2e-2 * 2.0 ** -22).all())


def test_moved_gradients_last_for_one_call_and_travel_with_a_capture(env):
    torch, binding = env
    n = 2300                                 # more pointers than one launch carries
    grads = [torch.full((3,), 1.0, device="cuda") for _ in range(n)]
    moved = [torch.full((3,), 1.0 + i, device="cuda") for i in range(n)]
    other = [torch.full((3,), -7.0, device="cuda") for i in range(n)]
    ps = [torch.zeros(3, device="cuda") for _ in range(n)]
    opt = binding.AdamWOptimizer(ps, grads)
    one = dict(lr=0.0, beta1=0.0, beta2=0.0)                 # m is the gradient
    opt.step(**one, grads=moved)
    assert torch.equal(torch.stack(opt.m), torch.stack(moved))
    opt.step(**one)
    assert torch.equal(torch.stack(opt.m), torch.stack(grads))
    graphs = []
    for g in (moved, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            opt.step(**one, grads=g)
        graphs.append((graph, g))
    for k in (0, 1, 0):
        graphs[k][0].replay()
        assert torch.equal(torch.stack(opt.m), torch.stack(graphs[k][1]))
        opt.step(**one, grads=grads)
        assert torch.equal(torch.stack(opt.m), torch.stack(grads))


def test_norm_clip_and_step_together(env):
    """The coefficient of the clipping goes from kernel to kernel."""
    torch, binding = env
    grads = [torch.randn(n, device="cuda") for n in (5000, 300)]
    ps = [torch.zeros_like(g) for g in grads]
    clip, opt = binding.GradClip(grads), binding.AdamWOptimizer(ps, grads)
    _, coef, _ = clip.norm(0.5)
    opt.step(lr=0.0, beta1=0.0, device_scale=coef)
    for g, m in zip(grads, opt.m):
        assert torch.equal(m, g * coef)


def test_another_stream_and_device_order(env):
    torch, binding = env
    g = torch.randn(1 << 22, device="cuda")
    p = torch.zeros_like(g)
    opt = binding.AdamWOptimizer([p], [g])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g.mul_(2.0)
        opt.step(lr=0.0, beta1=0.0)
        m = opt.m[0].clone()
    side.synchronize()
    assert torch.equal(m, g)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_two_to_the_31_elements(env, bits):
    """The last elements are those of a small tensor whose blocks have the same numbers (the random bits go by them)."""
    torch, binding = env
    n, tail = (1 << 31) + 300, 300
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-tail:] = torch.randn(tail, device="cuda").bfloat16()
    opt = binding.AdamWOptimizer([p], [g], state_bits=bits, seed=4)
    opt.step(lr=1e-2)
    assert not p[:-tail].any()
    m, v = ref.step(np.zeros(tail, np.float32), g[-tail:].float().cpu().numpy(), np.zeros(tail, np.float32), np.zeros(tail, np.float32), dict(HP, weight_decay=0.0), 1)[1:3]
    if bits == 32:
        assert np.array_equal(opt.m[0][-tail:].cpu().numpy(), m) and np.array_equal(opt.v[0][-tail:].cpu().numpy(), v)
    else:                                # (2^31 is a multiple of 256: the tail begins a block)
        r = ref.random_bits(tail, (1 << 31) // 256, 4, 1)
        codes, scales = ref.encode(m, r & np.uint64(0xFFFF), ref.E4M3, 7, True)
        assert np.array_equal(opt.m[0].view(torch.uint8)[-tail:].cpu().numpy(), codes) and np.array_equal(opt.m_scale[0].view(torch.uint8)[-2:].cpu().numpy(), scales)
    want, _, _, tol = ref.step(np.zeros(tail, np.float32), g[-tail:].float().cpu().numpy(), np.zeros(tail, np.float32), np.zeros(tail, np.float32), dict(HP, weight_decay=0.0), 1)
    assert (np.abs(p[-tail:].cpu().numpy() - want) <= tol).all()


def test_refusals(env):
    torch, binding = env
    E = binding.CameError
    p, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    new = binding.AdamWOptimizer
    for bad, status in (
            (lambda: new([], []), 2), (lambda: new([p], [g, g]), 2), (lambda: new([p.cpu()], [g]), 7), (lambda: new([p], [g.cpu()]), 7),
            (lambda: new([p.half()], [g]), 3), (lambda: new([p], [g.half()]), 3), (lambda: new([p], [g[:63]]), 2), (lambda: new([p], [p]), 12),
            (lambda: new([p[::2]], [g[:32]]), 11), (lambda: new([p], [g], state_bits=4), 3), (lambda: new([p], [g], state_bits=[8, 8]), 2),
            (lambda: new([p], [g], m=[torch.zeros_like(p)]), 1), (lambda: new([p], [g], state_bits=8, m_scale=[p]), 1), (lambda: new([p], [g], flags=[2]), 11), (lambda: new([p], [g], seed=-1), 5),
            (lambda: new([p, p[10:20]], [g, g[:10]]), 12), (lambda: new([p], [g], bf16_copy=[g]), 3),
            (lambda: new([p], [g], state_bits=8, m=[torch.zeros(64, device="cuda").to(torch.float8_e4m3fn)],
                         v=[torch.zeros(64, device="cuda").to(torch.float8_e5m2)]), 1)):
        with pytest.raises(E) as e:
            bad()
        assert e.value.status == status, e.value
    opt = new([p], [g])
    for kw, status in ((dict(lr=-1.0), 5), (dict(lr=float("nan")), 5), (dict(lr=1.0, beta1=1.0), 5), (dict(lr=1.0, beta2=1 - 1e-12), 5),
                       (dict(lr=1.0, eps=-1.0), 5), (dict(lr=1.0, weight_decay=float("inf")), 5), (dict(lr=1.0, grad_scale=1e-60), 5),
                       (dict(lr=1.0, device_scale=torch.ones(2, device="cuda")), 2), (dict(lr=1.0, device_scale=torch.ones(1)), 7),
                       (dict(lr=1.0, device_step=torch.ones(1, device="cuda")), 3), (dict(lr=1.0, grads=[g, g]), 2),
                       (dict(lr=1.0, grads=[g.bfloat16()]), 3), (dict(lr=1.0, grads=[g[:5]]), 2)):
        with pytest.raises(E) as e:
            opt.step(**kw)
        assert e.value.status == status, (kw, e.value)
    assert opt.step_count == 0 and not p.any()


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_blocks_of_large_values(env, gdt):
    """Blocks of m up to 1e38 and of v up to 9e35 (larger gradients' squares overflow), whose scales lie at the end of their range."""
    sizes = [1e17, 1e18, 5e18, 1e19, 1.7e19, 1e20, 1e29, 1e30, 1e31, 1e33, 1e36, 3e38]
    pair = Pair(env, [256 * len(sizes) + 300], [0], gdt, 8)
    for _ in range(3):
        pair.new_gradients()
        for i, size in enumerate(sizes + [1e30]):        # (and a short block)
            part = pair.g[0][256 * i:256 * (i + 1)] if i < len(sizes) else pair.g[0][-40:]
            x = size * pair.rng.uniform(0.25, 1.0, part.numel()) * pair.rng.choice([-1.0, 1.0], part.numel())
            part.copy_(pair.torch.from_numpy(x.astype(np.float32)))
        pair.check_step()
        # a code of at least half of the block's largest is there: nothing has vanished
        assert all(int((pair.bytes_of(pair.m[0])[256 * i:256 * (i + 1)] & 127).max()) >= 0x70 for i in range(len(sizes)))


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_subnormal_second_moments_beside_larger_ones(env, gdt):
    """A v above zero is stored as something above zero, also where it is a subnormal number (here 2e-41 to 4e-40)."""
    pair = Pair(env, [1024, 300], [0, 0], gdt, 8)
    for _ in range(3):
        pair.new_gradients()
        for g in pair.g:
            x = pair.rng.uniform(1.5e-19, 6e-19, g[3::7].numel()) * pair.rng.choice([-1.0, 1.0], g[3::7].numel())
            g[3::7] = pair.torch.from_numpy(x.astype(np.float32)).to(device=g.device, dtype=g.dtype)
        pair.check_step()
        assert all((pair.bytes_of(v)[3::7] > 0).all() for v in pair.v)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-20, 1e-15, 5.7e-11, 5.8e-11])
def test_small_gradients_with_a_smaller_eps(env, bits, eps):
    """Gradients of 1e-20 to 1e-17: their second moments are subnormal numbers in the first steps, and count, with eps on both sides
    of the border from which on they are left out."""
    pair = Pair(env, [1024, 77], [0, 0], "f32", bits)
    for _ in range(3):
        for g in pair.g:
            x = 10.0 ** pair.rng.uniform(-20, -17, g.numel()) * pair.rng.choice([-1.0, 1.0], g.numel())
            g.copy_(pair.torch.from_numpy(x.astype(np.float32)))
        pair.check_step(dict(HP, eps=eps))
        assert all(bool(p.isfinite().all()) for p in pair.p)
