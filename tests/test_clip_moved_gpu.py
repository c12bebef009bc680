"""Gradients that are replaced between calls of one GradClip: in a stream capture, over outputs, and while
the GPU is busy."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _lists(torch, fills, sizes=(1000, 33, 4097)):
    """Lists of constant tensors: the norm of tensor i of a list filled with f is f * sqrt(size i)."""
    return [[torch.full((n,), float(f), device="cuda") for n in sizes] for f in fills]


def _is_norm_of(got, grads):
    """Small whole numbers: the sums are exact, the square roots are rounded once."""
    want = [float((g.double() ** 2).sum().sqrt().float()) for g in grads]
    return got[2].tolist() == want


def test_a_replacement_inside_a_capture_is_refused(env):
    """A captured copy of the addresses runs at replay only: the context must not take it as done."""
    torch, binding = env
    a, b, c = _lists(torch, (1, 2, 4))
    clip = binding.GradClip(a)
    clip.norm(grads=b)
    clip.norm(grads=a)
    torch.cuda.synchronize()
    graph, refused = torch.cuda.CUDAGraph(), None
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        clip.norm(grads=a)                               # the same addresses: nothing to copy
        try:
            clip.norm(grads=b)
        except binding.CameError as e:
            refused = e.status
    assert _is_norm_of(clip.norm(grads=b), b)
    assert _is_norm_of(clip.norm(grads=c), c)
    assert refused == binding.CAME_ERR_UNSUPPORTED
    assert clip.grads[0] is c[0]
    clip.tensor_norms.zero_()
    graph.replay()                                       # reads the gradients that the context holds now
    torch.cuda.synchronize()
    assert _is_norm_of((None, None, clip.tensor_norms), c)
    assert _is_norm_of(clip.norm(grads=a), a)


def test_the_first_replacement_inside_a_capture_is_refused(env):
    torch, binding = env
    a, b = _lists(torch, (1, 2))
    clip = binding.GradClip(a)
    clip.norm()
    torch.cuda.synchronize()
    refused = None
    with torch.cuda.graph(torch.cuda.CUDAGraph(), capture_error_mode="relaxed"):
        clip.norm()
        try:
            clip.norm(grads=b)
        except binding.CameError as e:
            refused = e.status
    assert refused == binding.CAME_ERR_UNSUPPORTED
    assert _is_norm_of(clip.norm(), a) and _is_norm_of(clip.norm(grads=b), b)


def test_a_replacement_that_meets_an_output_is_refused(env):
    """Blocks that write one tensor's output must not race with blocks that read another's gradient."""
    torch, binding = env
    buf = torch.zeros(4 * 8192, device="cuda")
    g, fresh = _lists(torch, (1, 2), sizes=(5000, 5000))
    outs = [buf[:5000], buf[8192:13192]]

    def refused(clip, grads):
        for call in (lambda: clip.clip(1.0, grads=grads), lambda: clip.norm(1.0, grads=grads)):
            with pytest.raises(binding.CameError) as e:
                call()
            assert e.value.status == binding.CAME_ERR_OVERLAP
            assert clip.grads[0] is g[0]

    clip = binding.GradClip(g, outs)
    refused(clip, [outs[1], outs[0]])                    # each over the other's output
    refused(clip, [buf[8:5008], g[1]])                   # eight elements into its own output
    refused(clip, [g[0], buf[13191:18191]])              # the last element of an output
    assert bool((buf == 0).all())
    _, coef, _ = clip.clip(1.0)                          # the context still works, on the gradients that it had
    assert torch.equal(outs[0], g[0] * coef) and torch.equal(outs[1], g[1] * coef)
    _, coef, _ = clip.clip(1.0, grads=fresh)
    assert torch.equal(outs[0], fresh[0] * coef) and torch.equal(outs[1], fresh[1] * coef)
    old = outs[0].clone()                                # exactly its own output: in place
    _, coef, _ = clip.clip(0.5, grads=[outs[0], fresh[1]])
    assert torch.equal(outs[0], old * coef) and torch.equal(outs[1], fresh[1] * coef)
    _, coef, _ = clip.clip(1.0, grads=[g[0], buf[13192:18192]])          # right behind an output
    assert torch.equal(outs[0], g[0] * coef) and bool((outs[1] == 0).all())

    clip = binding.GradClip(g, g)                        # in place: the outputs move with the gradients
    refused(clip, [buf[:5000], buf[3000:8000]])
    halves = [buf[16384:21384], buf[21384:26384]]
    for h in halves:
        h.fill_(3.0)
    _, coef, _ = clip.clip(1.0, grads=halves)
    assert all(torch.equal(h, torch.full_like(h, 3.0) * coef) for h in halves)

    wide = torch.ones(5000, device="cuda")               # in place, but another type
    clip = binding.GradClip(g, [wide.view(torch.bfloat16)[:5000], torch.empty(5000, device="cuda", dtype=torch.bfloat16)])
    refused(clip, [wide, g[1]])
    assert bool((wide == 1).all())
    clip = binding.GradClip(g)                           # without outputs nothing can meet
    assert _is_norm_of(clip.norm(grads=[wide, wide]), [wide, wide])


def test_replacements_do_not_wait_for_the_gpu(env):
    """Two calls whose gradients have moved return while the stream still works on what came before."""
    torch, binding = env
    a, b = _lists(torch, (1, 2))
    clip = binding.GradClip(a)
    clip.norm(grads=b)
    clip.norm(grads=a)
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    torch.cuda._sleep(1_000_000_000)                     # half a second
    done.record()
    clip.norm(grads=b)
    clip.norm(grads=a)
    assert not done.query()
    for k in range(9):                                   # every call finds the addresses that it was given
        now = b if k % 2 else a
        assert _is_norm_of(clip.norm(grads=now), now)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("count", [1, 600])
def test_outputs_of_moved_gradients(env, dtype, count):
    """Gradients that move to other alignments than their outputs and back: written wide, one by one, wide.
    count tensors: the list's sums are finished in one stage, or in two."""
    torch, binding = env
    dtype = getattr(torch, dtype)
    sizes = [4097, 300, 8192][:max(1, min(3, count))] * max(1, count // 3)
    flat = torch.empty(sum(sizes) + 16 * len(sizes), device="cuda", dtype=dtype)

    def views(flat, shift):
        at, got = 0, []
        for n in sizes:
            got.append(flat[at + shift:at + shift + n])
            at += n // 8 * 8 + 16
        return got

    outs = views(torch.empty_like(flat), 0)
    clip = binding.GradClip([g.normal_() for g in views(flat, 0)], outs)
    for shift in (0, 1, 7, 8, 2, 0):
        grads = views(torch.randn(flat.numel(), device="cuda").to(dtype), shift)
        total, coef, _ = clip.clip(0.25, grads=grads)
        want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
        assert abs(float(total) - want) <= 2.5e-6 * want                 # 64 * 2^-24 / 2 of a sum of squares, and its rounding
        assert all(torch.equal(o, (g.float() * coef).to(dtype)) for o, g in zip(outs, grads))
