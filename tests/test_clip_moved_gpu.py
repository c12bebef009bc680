"""Gradients that are replaced between calls of one GradClip: what a stream capture may hold."""
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
