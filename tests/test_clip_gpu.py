"""Global gradient norm and clipping against the formulas in 64 bits, and the step that takes the
coefficient from device memory.

Tolerances, from the arithmetic: a thread adds at most a few dozen fp32 squares here before it
goes on in double, each addition rounds by 2^-24, all terms are positive: relative error of a sum
of squares below 64 * 2^-24, of a norm below half of that, plus its own rounding to fp32:
NORM_TOL = 2.5e-6.  The coefficient inherits that.  An output is fl(g * fl(s * coef)) and is checked
bit for bit given the coefficient, and to NORM_TOL + 3 * 2^-24 (fp32) or + 2^-8 (bf16) in all."""
import numpy as np
import pytest

from paper_2307_02047_b200 import synth

pytestmark = pytest.mark.gpu
NORM_TOL = 2.5e-6
SENT = 1232.0


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _dt(torch, name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _guarded(torch, n, dtype, offset, fill=SENT):
    """A view of n elements, `offset` elements after a 256-byte boundary, inside a guarded buffer."""
    arena = torch.full((128 + offset + n + 128,), fill, dtype=dtype, device="cuda")
    assert arena.data_ptr() % 256 == 0
    return arena, arena[128 + offset:128 + offset + n]


def _check(torch, grads, sizes, got, max_norm, eps, s):
    """Norms and coefficient against float64."""
    total, coef, each = (x.double().cpu().numpy() for x in got)
    want = np.array([np.sqrt(np.sum(np.square(g.double().cpu().numpy()))) * s for g in grads])
    N = float(np.sqrt(np.sum(want ** 2)))
    np.testing.assert_allclose(each, want, rtol=NORM_TOL, atol=0)
    np.testing.assert_allclose(total, N, rtol=NORM_TOL, atol=0)
    c = 1.0 if N + eps <= max_norm else max_norm / (N + eps)
    np.testing.assert_allclose(coef, c, rtol=NORM_TOL, atol=0)
    return N, c


LISTS = [
    ([1], [0]), ([0], [0]), ([0, 5, 0], [0, 3, 0]), ([7, 8, 9, 15, 16, 17], [0, 1, 2, 3, 4, 5]),
    ([31, 32, 33, 255, 256, 257], [1, 0, 7, 15, 9, 8]), ([4095, 4096, 4097, 8192, 8193], [0, 0, 1, 13, 0]),
    ([513 * 1030, 1001, 65 * 33, 1, 7, 300], [0, 3, 1, 0, 5, 0]), ([3_000_001], [1]), ([100] * 700, [0] * 700),
]


@pytest.mark.parametrize("gdt,odt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("k", range(len(LISTS)))
def test_norm_and_clip_against_64_bits(env, gdt, odt, k):
    torch, binding = env
    sizes, offs = LISTS[k]
    gen = torch.Generator(device="cuda").manual_seed(11 + k)
    grads, outs, arenas = [], [], []
    for i, (n, o) in enumerate(zip(sizes, offs)):
        a, g = _guarded(torch, n, _dt(torch, gdt), o)
        g.normal_(0, 10.0 ** (-1 - i % 4), generator=gen)
        b, out = _guarded(torch, n, _dt(torch, odt), o if i % 3 else o + 1)      # also other offsets than the gradient's
        grads.append(g); outs.append(out); arenas.append((b, 128 + (o if i % 3 else o + 1), n))
        arenas.append((a, 128 + o, n))
    before = [g.clone() for g in grads]
    clip = binding.GradClip(grads, outs)
    for max_norm, eps, s in ((0.05, 1e-6, 1.0), (1e9, 0.0, 0.25), (float("inf"), 1e-6, 3.0)):
        got = clip.clip(max_norm, eps, s)
        N, c = _check(torch, grads, sizes, got, max_norm, eps, s)
        f = torch.tensor(np.float32(s), device="cuda") * clip.coef
        for g, out, old in zip(grads, outs, before):
            assert torch.equal(g, old)
            assert torch.equal(out, (g.float() * f).to(out.dtype))
            want = old.double().cpu().numpy() * (s * c)
            tol = NORM_TOL + (3 * 2.0 ** -24 if odt == "f32" else 2.0 ** -8)
            np.testing.assert_allclose(out.double().cpu().numpy(), want, rtol=tol, atol=1e-37)
        for arena, at, n in arenas:
            assert bool((arena[:at] == SENT).all()) and bool((arena[at + n:] == SENT).all())


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_clip_in_place_and_untouched_when_small(env, gdt):
    torch, binding = env
    grads = [torch.randn(n, device="cuda").to(_dt(torch, gdt)) for n in (1000, 33, 4097)]
    before = [g.clone() for g in grads]
    clip = binding.GradClip(grads, grads)
    clip.clip(1e6)
    assert float(clip.coef) == 1.0 and all(torch.equal(a, b) for a, b in zip(grads, before))
    clip.clip(0.5)
    f = clip.coef.clone()
    assert 0 < float(f) < 1
    for a, b in zip(grads, before):
        assert torch.equal(a, (b.float() * f).to(b.dtype))
    # moved gradients: clipped where they now are
    fresh = [b.clone() for b in before]
    kept = [g.clone() for g in grads]
    clip.clip(0.5, grads=fresh)
    assert torch.equal(clip.coef, f)
    for a, b, old, k in zip(fresh, before, grads, kept):
        assert torch.equal(a, (b.float() * f).to(b.dtype)) and torch.equal(old, k)


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_large_small_and_non_finite_values(env, gdt):
    torch, binding = env
    dt = _dt(torch, gdt)
    big = torch.full((5003,), 3e25, dtype=dt, device="cuda")          # its square overflows fp32
    ones = torch.ones(77, dtype=dt, device="cuda")
    clip = binding.GradClip([ones, big])
    _check(torch, [ones, big], None, clip.norm(1.0), 1.0, 1e-6, 1.0)
    # finite elements whose norm passes fp32: N = inf, coef still what the formula gives
    huge = torch.full((64,), 3e38, dtype=dt, device="cuda")
    n, c, _ = binding.GradClip([huge]).norm(1.0, eps=0.0)
    assert float(n) == float("inf")
    want = 1.0 / (8.0 * huge[0].double().item())
    assert abs(float(c) - want) <= 2e-6 * want + 2.0 ** -149
    for bad, isnan in ((float("inf"), False), (float("-inf"), False), (float("nan"), True)):
        for at in (0, 76, 40):
            x = ones.clone()
            x[at] = bad
            out = torch.empty_like(x)
            clip = binding.GradClip([ones, x], [torch.empty_like(ones), out])
            n, c, each = clip.clip(1.0)
            assert abs(float(each[0]) - 77 ** 0.5) < 1e-5
            assert (n.isnan() and c.isnan() and each[1].isnan()) if isnan else (n.isinf() and float(c) == 0 and each[1].isinf())
            assert torch.equal(out.isnan(), torch.arange(77, device="cuda").eq(at) | isnan)
    zero = torch.zeros(1000, dtype=dt, device="cuda")
    n, c, each = binding.GradClip([zero]).norm(1.0, eps=0.0)
    assert float(n) == 0 and float(c) == 1 and float(each[0]) == 0


def test_more_than_two_to_the_31_elements(env):
    torch, binding = env
    n = (1 << 31) + 17
    g = torch.full((n + 3,), 0.5, dtype=torch.bfloat16, device="cuda")[3:]
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    norm, coef, _ = binding.GradClip([g], [out]).clip(0.25 * n ** 0.5)
    assert abs(float(norm) - 0.5 * n ** 0.5) <= NORM_TOL * 0.5 * n ** 0.5
    want = (0.5 * coef).bfloat16()
    assert bool((out[:1000] == want).all()) and bool((out[-1000:] == want).all())
    assert int((out == want).sum()) == n


def test_results_do_not_depend_on_timing_or_stream(env):
    torch, binding = env
    g = [torch.randn(n, device="cuda") for n in (5_000_003, 17, 1_000_000)]
    clip = binding.GradClip(g)
    clip.norm(1.0)
    first = clip.results.clone()
    side = torch.cuda.Stream()
    for k in range(20):
        with torch.cuda.stream(side if k % 2 else torch.cuda.current_stream()):
            side.wait_stream(torch.cuda.default_stream())
            clip.norm(1.0)
        torch.cuda.synchronize()
        assert torch.equal(clip.results, first)


def test_capture_and_replay(env):
    torch, binding = env
    g = [torch.randn(n, device="cuda") for n in (100_003, 17)]
    out = [torch.empty_like(x) for x in g]
    clip = binding.GradClip(g, out)
    clip.clip(1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip.clip(1.0)
    for x in g:
        x.mul_(3.0)
    graph.replay()
    f = clip.coef.clone()
    torch.cuda.synchronize()
    replayed = [o.clone() for o in out]
    clip.clip(1.0)
    assert torch.equal(clip.coef, f) and all(torch.equal(a, b) for a, b in zip(replayed, out))


@pytest.mark.parametrize("schedule", [1, 2])
@pytest.mark.parametrize("adafactor", [False, True])
@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_step_takes_the_coefficient_from_device_memory(env, schedule, adafactor, gdt):
    """A step scaled on the device equals, bit for bit, a step whose grad_scale is that number."""
    torch, binding = env
    shapes = [(257, 1032), (33, 65), (300, 1), (1001,)]
    hp = dict(synth.PAPER_HPARAMS, weight_decay=0.01)
    torch.manual_seed(3)
    p0 = [torch.randn(s, device="cuda") * 0.02 for s in shapes]
    steps = [[(torch.randn(s, device="cuda") * 1e-2).to(_dt(torch, gdt)) for s in shapes] for _ in range(3)]
    flags = binding.CAME_CREATE_ADAFACTOR if adafactor else 0
    binding.came_tune(binding.CAME_TUNE_SCHEDULE, schedule)
    try:
        sides = []
        for device_side in (True, False):
            p = [x.clone() for x in p0]
            g = [x.clone() for x in steps[0]]
            opt = binding.CameOptimizer(p, g, create_flags=flags)
            clip = binding.GradClip(g)
            for fresh in steps:
                for a, b in zip(g, fresh):
                    a.copy_(b)
                _, coef, _ = clip.norm(0.25)
                assert 0 < float(coef) < 1
                if device_side:
                    opt.step(device_scale=coef, **hp)
                else:
                    opt.step(grad_scale=float(coef), **hp)
            torch.cuda.synchronize()
            sides.append(p + opt.m + opt.r)
            opt.close()
    finally:
        binding.came_tune(binding.CAME_TUNE_SCHEDULE, 0)
    assert all(torch.equal(a, b) for a, b in zip(*sides))


def test_refusals(env):
    torch, binding = env
    g = [torch.ones(100, device="cuda")]

    def refused(status, call):
        with pytest.raises(binding.CameError) as e:
            call()
        assert e.value.status == status

    clip = binding.GradClip(g)
    refused(binding.CAME_ERR_UNSUPPORTED, lambda: clip.clip(1.0))
    for kw in (dict(max_norm=0.0), dict(max_norm=float("nan")), dict(max_norm=-1.0), dict(max_norm=1.0, eps=-1.0),
               dict(max_norm=1.0, eps=float("inf")), dict(max_norm=1.0, grad_scale=-2.0), dict(max_norm=1.0, grad_scale=float("nan"))):
        refused(binding.CAME_ERR_HPARAM, lambda: clip.norm(**kw))
    refused(binding.CAME_ERR_SHAPE, lambda: clip.norm(1.0, grads=g + g))
    refused(binding.CAME_ERR_SHAPE, lambda: clip.norm(1.0, grads=[torch.ones(99, device="cuda")]))
    refused(binding.CAME_ERR_SHAPE, lambda: clip.norm(1.0, grads=[torch.ones(100, device="cuda").bfloat16()]))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.GradClip([]))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.GradClip(g, [torch.ones(99, device="cuda")]))
    refused(binding.CAME_ERR_DTYPE, lambda: binding.GradClip([torch.ones(4, device="cuda", dtype=torch.float64)]))
    refused(binding.CAME_ERR_DEVICE, lambda: binding.GradClip([torch.ones(4)]))
    refused(binding.CAME_ERR_UNSUPPORTED, lambda: binding.GradClip([torch.ones(4, 4, device="cuda").t()[:2]]))
    refused(binding.CAME_ERR_OVERLAP, lambda: binding.GradClip([g[0][:50], g[0][40:90]], [g[0][:50], g[0][40:90]]))
    refused(binding.CAME_ERR_OVERLAP, lambda: binding.GradClip([g[0][:50]], [g[0][10:60]]))
    assert float(clip.norm(5.0)[1]) == pytest.approx(0.5)      # the context still works
    opt = binding.CameOptimizer([torch.ones(8, device="cuda")], [torch.ones(8, device="cuda")])
    refused(binding.CAME_ERR_DTYPE, lambda: opt.step(device_scale=torch.ones((), device="cuda").double(), **synth.PAPER_HPARAMS))
    refused(binding.CAME_ERR_SHAPE, lambda: opt.step(device_scale=torch.ones(2, device="cuda"), **synth.PAPER_HPARAMS))
    opt.step(**synth.PAPER_HPARAMS)
    opt.close()
