"""Pre-scales at the ends of fp32's range: clipped outputs are products with the fp32 value, norms are not."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e39, 1e300, 1e-46, 1e-300])
def test_a_pre_scale_that_fp32_does_not_hold_is_refused_for_outputs(scale):
    import torch
    from paper_2307_02047_b200 import binding
    out = torch.full((1000,), 7.0, device="cuda")
    clip = binding.GradClip([torch.zeros(1000, device="cuda")], [out])
    with pytest.raises(binding.CameError) as e:          # infinity would make NaN of these zeros
        clip.clip(1.0, grad_scale=scale)
    assert e.value.status == binding.CAME_ERR_HPARAM and bool((out == 7).all())
    assert clip.norm(1.0, grad_scale=scale)[0].item() == 0.0             # computed in double


@pytest.mark.parametrize("scale,size", [(1e39, 1e-30), (1e-46, 1e30), (3e38, 1e-20), (1e-40, 1e20)])
def test_norms_take_any_pre_scale(scale, size):
    """One value n times: the squares round in fp32, 64 additions at most do, and the norm to fp32."""
    import torch
    from paper_2307_02047_b200 import binding
    g = torch.full((1000,), size ** 0.5, device="cuda")
    want = float(g[0].double()) * scale * 1000 ** 0.5
    n = float(binding.GradClip([g]).norm(float("inf"), grad_scale=scale)[0])
    assert abs(n - want) <= 2.5e-6 * want
