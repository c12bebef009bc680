"""The lookup's gradient where a warp has more than 32 sorted tokens, as training batches of wide models do.

Whole numbers small enough that every sum is exact in fp32, whatever its order: the fp32 result equals
the one in 64 bits, the bf16 result is that one rounded."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _ids(torch, kind, tokens, rows, gen):
    if kind == "same":
        return torch.full((tokens,), rows // 2, device="cuda")
    if kind == "hot":                        # frequencies that fall as 1 / rank
        u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
        return (torch.exp(u * torch.log(torch.tensor(rows + 1.0, dtype=torch.float64))) - 1).long().clamp_(0, rows - 1)
    ids = torch.randint(0, rows, (tokens,), generator=gen, device="cuda")
    if kind == "padded":                     # three of four tokens are no rows: warps whose later groups are empty
        ids[torch.rand(tokens, generator=gen, device="cuda") < 0.75] = -1
    return ids


@pytest.mark.parametrize("tokens,cols,gap,kind,rows", [
    (70_001, 4096, 0, "hot", 32_000),        # 64 tokens per warp; 8 columns per access
    (70_001, 4096, 0, "any", 300),           # runs of 233
    (70_001, 4095, 0, "hot", 32_000),        # one column per access
    (70_001, 4092, 4, "padded", 5_000),      # four
    (65_600, 4096, 0, "any", 60_000),        # runs of one
    (65_536, 4096, 0, "same", 7),            # one run across all blocks
    (270_000, 4096, 0, "hot", 32_000),       # 128 per warp
    (270_007, 4095, 1, "any", 1_000),
    (270_007, 4096, 0, "padded", 200_000),
])
@pytest.mark.parametrize("ydt,gdt", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32"), ("float32", "bfloat16")])
def test_every_group_of_a_warp_is_added(env, tokens, cols, gap, kind, rows, ydt, gdt):
    torch, binding = env
    gen = torch.Generator(device="cuda").manual_seed(tokens + cols)
    ids = _ids(torch, kind, tokens, rows, gen)
    ids = ids.int() if rows % 2 else ids
    draw = lambda n: torch.randint(-3, 4, (n, cols + gap), generator=gen, device="cuda", dtype=torch.int8)  # noqa: E731
    dy = draw(tokens).to(getattr(torch, ydt))[:, :cols]
    for accumulate in (False, True):
        grad = draw(rows).to(getattr(torch, gdt))[:, :cols]
        old = grad.clone()
        binding.embed_backward(dy, ids, grad, 2.0, accumulate=accumulate)
        ok = (ids >= 0).nonzero()[:, 0]
        for a in range(0, cols, 1024):       # the reference in 64 bits, by columns
            part = slice(a, min(cols, a + 1024))
            want = old[:, part].double() if accumulate else torch.zeros_like(old[:, part], dtype=torch.float64)
            want.index_add_(0, ids[ok].long(), 2.0 * dy[ok, part].double())
            assert float(want.abs().max()) < 2 ** 24
            assert torch.equal(grad[:, part], want.to(grad.dtype))


def test_runs_across_many_blocks_are_joined_alike_every_time(env):
    """Three rows that share all blocks, many times over: the block that arrives last always finds
    the others' parts."""
    torch, binding = env
    tokens, rows, cols = 40_000, 3, 4096
    gen = torch.Generator(device="cuda").manual_seed(6)
    ids = torch.randint(0, rows, (tokens,), generator=gen, device="cuda")
    grad = torch.empty(rows, cols, device="cuda")
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(10):
        dy = torch.randint(-3, 4, (tokens, cols), generator=gen, device="cuda", dtype=torch.int8)
        want = torch.stack([dy[ids == v].sum(0) for v in range(rows)]).float()
        dy = dy.bfloat16()
        for _ in range(30):
            wrong += (binding.embed_backward(dy, ids, grad) != want).sum()
    assert int(wrong) == 0
