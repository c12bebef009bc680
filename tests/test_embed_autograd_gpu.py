"""The lookup on a table that requires grad, and shapes that do not fit."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


@pytest.mark.parametrize("tdt,odt", [("float32", None), ("float32", "bfloat16"), ("bfloat16", None), ("bfloat16", "float32")])
@pytest.mark.parametrize("idt", ["int32", "int64"])
def test_the_table_gets_its_gradient(env, tdt, odt, idt):
    """Small whole numbers: sums and products are exact in fp32 and, below 256, in bf16."""
    torch, binding = env
    rows, cols = 50, 24
    table = torch.randint(-3, 4, (rows, cols), device="cuda").to(getattr(torch, tdt)).requires_grad_()
    ids = torch.randint(-1, rows + 1, (4, 31), device="cuda").to(getattr(torch, idt))
    out_dtype = getattr(torch, odt) if odt else None
    out = binding.embed_forward(table, ids, 2.0, out_dtype=out_dtype)
    with torch.no_grad():
        plain = binding.embed_forward(table, ids, 2.0, out_dtype=out_dtype)
    assert out.requires_grad and not plain.requires_grad and torch.equal(out.detach(), plain)
    dy = torch.randint(-2, 3, out.shape, device="cuda").to(out.dtype)
    out.backward(dy)
    ok = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    want.index_add_(0, ids[ok].long(), 2.0 * dy[ok].double())
    assert table.grad.dtype == table.dtype and torch.equal(table.grad.double(), want)
    binding.embed_forward(table, ids, 2.0).float().sum().backward()      # a gradient without memory of its own, and a second one added
    want.index_add_(0, ids[ok].long(), torch.full((int(ok.sum()), cols), 2.0, dtype=torch.float64, device="cuda"))
    assert torch.equal(table.grad.double(), want)


def test_what_has_no_gradient_is_refused(env):
    torch, binding = env
    table = torch.ones(5, 8, device="cuda", requires_grad=True)
    ids = torch.tensor([1, 2, 2], device="cuda")
    with pytest.raises(binding.CameError) as e:          # a buffer of the caller's has no graph
        binding.embed_forward(table, ids, out=torch.empty(3, 8, device="cuda"))
    assert e.value.status == binding.CAME_ERR_UNSUPPORTED
    out = torch.empty(3, 8, device="cuda")
    with torch.no_grad():
        assert binding.embed_forward(table, ids, out=out) is out
    assert binding.embed_forward(table.detach(), ids, out=out) is out and not out.requires_grad
    (g,) = torch.autograd.grad(binding.embed_forward(table, ids).square().sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):                    # once differentiable
        g.sum().backward()


def test_shapes_that_do_not_fit_are_refused_as_errors_of_the_library(env):
    torch, binding = env
    t, ids = torch.ones(10, 8, device="cuda"), torch.zeros(4, 3, device="cuda", dtype=torch.int64)
    crossed = torch.ones(3, 4, 8, device="cuda").transpose(0, 1)         # rows at two strides

    def refused(status, call):
        with pytest.raises(binding.CameError) as e:
            call()
        assert e.value.status == status

    refused(binding.CAME_ERR_UNSUPPORTED, lambda: binding.embed_forward(t, ids, out=crossed))
    refused(binding.CAME_ERR_UNSUPPORTED, lambda: binding.embed_backward(crossed, ids, t))
    one = torch.ones((), device="cuda")
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_forward(t, ids[0, 0], out=one))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(one, ids[0, 0], t))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(torch.ones(4, 3, 0, device="cuda"), ids, torch.ones(10, 0, device="cuda")))
    none = torch.ones(0, 3, 8, device="cuda")            # no tokens: any strides
    assert bool((binding.embed_backward(none, ids[:0], t.clone()) == 0).all())
    assert bool((t == 1).all())
