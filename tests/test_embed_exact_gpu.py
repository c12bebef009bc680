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


@pytest.mark.parametrize("cols", [1, 2, 4, 8, 72])
def test_subnormal_values_when_adding(env, cols):
    """Adding in fp32 takes subnormal old values, addends and results as zero (each below 2^-126): three of
    those at most, so the result is within 3 * 2^-126; what is overwritten, or bf16, keeps them.  Rows without
    tokens are not touched at all."""
    torch, binding = env
    values = [0.0, 1e-40, -1e-39, 1.1e-38, -1.2e-38, 1.5e-38, -1.4e-38, 1e-30]
    pairs = [(a, b) for a in values for b in values]
    old, new = (torch.tensor([p[k] for p in pairs] + [1e-40], device="cuda")[:, None].expand(-1, cols).contiguous() for k in (0, 1))
    ids = torch.arange(len(pairs), device="cuda")
    got = binding.embed_backward(new[:-1], ids, old.clone(), accumulate=True)
    assert float((got.double() - old.double() - new.double())[:-1].abs().max()) <= 3 * 2.0 ** -126
    assert torch.equal(got[-1], old[-1])
    assert torch.equal(binding.embed_backward(new[:-1], ids, old.clone())[:-1], new[:-1])
    narrow = old.bfloat16()
    got = binding.embed_backward(new[:-1], ids, narrow.clone(), accumulate=True)
    assert torch.equal(got[:-1], (narrow.float() + new).bfloat16()[:-1]) and torch.equal(got[-1], narrow[-1])
