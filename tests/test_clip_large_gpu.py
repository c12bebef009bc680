"""The gradient norm and clipping where tiles are large: the kernels that serve whole models.

Sets of more than 155 MB have tiles from 128 KB on, sets of more than 620 MB tiles of 512 KB."""
import pytest

pytestmark = pytest.mark.gpu
NORM_TOL = 2.5e-6                       # 64 additions in fp32 at most, then double: 64 * 2^-24 / 2, and the rounding to fp32


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def test_small_values_behind_large_ones_are_not_lost(env):
    """In every 512 KB four of sixteen elements of the first 4096 are 4096, the others of them 0, the rest 1: a
    thread that added all its squares to one fp32 number would stop at 2^24 (there 1 is half a
    spacing) and come out low by 7.5e-6, beyond the tolerance that its sum has at 64 additions."""
    torch, binding = env
    n, count = 262144, 1221             # 640 MB of bf16
    g = torch.ones(count, n, dtype=torch.bfloat16, device="cuda")
    g[:, :4096] = 0
    g.view(count, n // 16, 16)[:, :256, :4] = 4096
    got = binding.GradClip([g]).norm()[0]
    want = (count * (1024 * 4096.0 ** 2 + (n - 4096))) ** 0.5
    assert abs(float(got) - want) <= NORM_TOL * want


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_no_one_sided_error_on_normal_values(env, dtype):
    """Chains of up to 32 squares of normal values in fp32 come out low by 2e-8 of their sum (bf16; a
    thousand times less in fp32), what is left of 1e5 chains' random errors is below 1e-9: the norm is
    within 1e-8, its rounding to fp32 within 2^-24.  Chains of 256 would be low by 1.3e-7 and more."""
    torch, binding = env
    n = 330_000_000 if dtype == "bfloat16" else 160_000_000              # 640 MB and more
    g = torch.empty(n, dtype=getattr(torch, dtype), device="cuda").normal_(0, 1e-3, generator=torch.Generator(device="cuda").manual_seed(1))
    got = float(binding.GradClip([g]).norm()[0])
    want = sum(float((p.double() ** 2).sum()) for p in g.split(1 << 26)) ** 0.5
    assert abs(got - want) <= (2.0 ** -24 + 1e-8) * want


def _views(torch, sizes, offsets, dtype):
    """Tensors of one flat buffer, each `offset` elements behind a 64-byte boundary."""
    at, starts = 0, []
    for n, o in zip(sizes, offsets):
        starts.append(at + o)
        at += -(-(n + o) // 32) * 32
    flat = torch.zeros(at, dtype=getattr(torch, dtype), device="cuda")
    return flat, [flat[s:s + n] for s, n in zip(starts, sizes)]


SIZES = {   # elements; tiles of 128 KB and of 512 KB
    "fp32, 128 KB": ("float32", [20_000_003, 5, 19_000_001, 1000, 3 * 32768 + 1, 0, 7_123_457]),
    "bf16, 128 KB": ("bfloat16", [40_000_003, 5, 38_000_001, 1000, 3 * 65536 + 1, 0, 7_123_457]),
    "fp32, 512 KB": ("float32", [90_000_003, 5, 60_000_001, 1000, 3 * 131072 + 1, 0, 7_123_457]),
    "bf16, 512 KB": ("bfloat16", [190_000_003, 5, 120_000_001, 1000, 3 * 262144 + 1, 0, 7_123_457]),
}
OFFSETS = [3, 0, 17, 1, 31, 5, 8]


@pytest.mark.parametrize("odt", ["float32", "bfloat16", "in place"])
@pytest.mark.parametrize("case", list(SIZES))
def test_large_lists_of_odd_tensors(env, case, odt):
    """Norms against 64 bits; outputs bit for bit given the coefficient."""
    torch, binding = env
    dtype, sizes = SIZES[case]
    flat, grads = _views(torch, sizes, OFFSETS, dtype)
    gen = torch.Generator(device="cuda").manual_seed(len(odt))
    for i, g in enumerate(grads):
        g.normal_(0, 10.0 ** (-1 - i % 3), generator=gen)
    before = flat.clone()
    if odt == "in place":
        out_flat, outs = flat, grads
    else:                                    # every other output at another offset than its gradient
        out_flat, outs = _views(torch, sizes, [o + i % 2 for i, o in enumerate(OFFSETS)], odt)
    old = [before[g.storage_offset():g.storage_offset() + g.numel()] for g in grads]
    want = [sum(float((p.double() ** 2).sum()) for p in g.split(1 << 26)) ** 0.5 if g.numel() else 0.0 for g in grads]
    N = sum(w * w for w in want) ** 0.5
    total, coef, each = binding.GradClip(grads, outs).clip(0.5, 0.0)
    assert abs(float(total) - N) <= NORM_TOL * N
    assert abs(float(coef) - 0.5 / N) <= NORM_TOL * 0.5 / N
    for got, w in zip(each.tolist(), want):
        assert abs(got - w) <= NORM_TOL * w
    for o, g in zip(outs, old):
        for p, q in zip(o.split(1 << 26), g.split(1 << 26)):
            assert torch.equal(p, (q.float() * coef).to(o.dtype))
    if odt != "in place":
        assert torch.equal(flat, before)
    gaps = torch.ones(out_flat.numel(), dtype=torch.bool, device="cuda")
    for o in outs:
        gaps[o.storage_offset():o.storage_offset() + o.numel()] = False
    assert bool((out_flat[gaps] == 0).all())


@pytest.mark.parametrize("case", list(SIZES))
def test_every_element_counts_once(env, case):
    """Tensors of zeros with a few ones, at their ends, around the borders of tiles and anywhere: a norm is
    the square root of their number, exactly, and one that is missed or counted twice changes it."""
    torch, binding = env
    dtype, sizes = SIZES[case]
    flat, grads = _views(torch, sizes, OFFSETS, dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    counts = []
    for g in grads:
        if g.numel():
            at = [torch.tensor([0, g.numel() - 1], device="cuda")]
            tile = 16 * 1024                 # borders of tiles are among its multiples, counted from the start or the first aligned element
            border = torch.randint(0, g.numel() // tile + 1, (40,), generator=gen, device="cuda") * tile
            at += [border + k for k in range(-33, 34)] + [torch.randint(0, g.numel(), (200,), generator=gen, device="cuda")]
            at = torch.cat(at)
            g[at[(at >= 0) & (at < g.numel())]] = 1
        counts.append(int(g.count_nonzero()))
    total, coef, each = binding.GradClip(grads).norm()
    assert each.tolist() == torch.tensor(counts, dtype=torch.float64).sqrt().float().tolist()
    assert float(total) == float(torch.tensor(float(sum(counts)), dtype=torch.float64).sqrt().float())
    assert float(coef) == 1


def test_sums_of_many_tiles_and_tensors_are_finished_alike_every_time(env):
    """Whole numbers, so sums are exact: the tile and the tensor that arrive last always find the others'."""
    torch, binding = env
    sizes = [3_000_001, 17, 1_000_000] * 40  # two stages: above 64 tensors
    flat = torch.empty(sum(sizes), device="cuda")
    grads = list(flat.split(sizes))
    clip = binding.GradClip(grads)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(10):
        flat.copy_(torch.randint(-2, 3, flat.shape, device="cuda", dtype=torch.int8))
        want = torch.stack([(g.double() ** 2).sum() for g in grads]).sqrt().float()
        all_ = (flat.double() ** 2).sum().sqrt().float()
        for _ in range(100):
            total, _, each = clip.norm()
            wrong += (each != want).sum() + (total != all_)
    assert int(wrong) == 0
