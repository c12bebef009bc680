"""Identities of the lookup and its gradient that hold exactly on small whole numbers."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


@pytest.mark.parametrize("tokens,rows,cols", [(1, 3, 8), (50, 20, 5), (400, 90, 72), (2000, 301, 136), (9000, 700, 64), (20_000, 40, 33)])
def test_gradient_equals_differences_exactly(env, tokens, rows, cols):
    """<dW, E> = <c, out(W + E) - out(W - E)> / 2 for every E, as the lookup is linear in the table.  Whole
    numbers up to 4: every product, sum and difference is a whole number below 2^24 in fp32 and
    below 2^53 in the inner products, so both sides are exact and equal.  E and c are positive, so a
    token left out or added twice changes the left side."""
    torch, binding = env
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    whole = lambda *s: torch.randint(-4, 5, s, generator=gen, device="cuda").float()  # noqa: E731
    ids = torch.randint(-1, rows + 1, (tokens,), generator=gen, device="cuda")
    ids[0] = rows - 1
    ok = (ids >= 0) & (ids < rows)
    scale = 4.0
    for _ in range(3):
        W, E = whole(rows, cols), torch.randint(1, 5, (rows, cols), generator=gen, device="cuda").float()
        c = torch.randint(1, 5, (tokens, cols), generator=gen, device="cuda").float()
        dW = binding.embed_backward(c, ids, torch.empty_like(W), scale)
        left = float((dW.double() * E.double()).sum())
        diff = binding.embed_forward(W + E, ids, scale).double() - binding.embed_forward(W - E, ids, scale).double()
        assert left == float((c.double() * diff).sum()) / 2
        # the same sum from the formula, and what any one token gives to it
        each = scale * (c[ok].double() * E[ids[ok]].double()).sum(1)
        assert left == float(each.sum()) and float(each.min()) > 0
