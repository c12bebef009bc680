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
