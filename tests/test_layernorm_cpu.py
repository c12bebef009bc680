"""Refusals of the layer norm's entry points that are decided before any CUDA call, and its workspace."""
import pytest

from paper_2307_02047_b200 import binding


def _l(**over):
    d = dict(x=0x100000, weight=0x200000, bias=0x210000, y=0x300000, dy=0x400000, dx=0x500000, dweight=0x600000, dbias=0x610000, mean=0x700000,
             rstd=0x710000, rows=10, cols=8, x_ld=8, y_ld=8, dx_ld=8, eps=1e-5, x_dtype=0, y_dtype=0, dx_dtype=0, weight_dtype=0, flags=0, reserved=0)
    d.update(over)
    return binding.came_layernorm(**d)


FORWARD, BACKWARD = (lambda l: binding.came_layernorm_forward(l)), (lambda l: binding.came_layernorm_backward(l, 0x800000, 1 << 20))


@pytest.mark.parametrize("over,status", [
    (dict(rows=-1), 2), (dict(rows=(1 << 30) + 1), 2), (dict(cols=0), 2), (dict(cols=(1 << 27) + 1), 2), (dict(x_ld=7), 2), (dict(y_ld=7), 2),
    (dict(x_ld=(1 << 29) + 1), 2), (dict(x_dtype=2), 3), (dict(y_dtype=-1), 3), (dict(weight_dtype=5), 3), (dict(flags=2), 11), (dict(reserved=1), 2),
    (dict(x=None), 1), (dict(x=0x100002), 4), (dict(weight=0x200001), 4), (dict(mean=0x700002), 4),
])
def test_refused_in_both_directions(over, status):
    for call in (FORWARD, BACKWARD, binding.came_layernorm_workspace):
        if call is FORWARD and "mean" in over:
            over = {**over}
        with pytest.raises(binding.CameError) as e:
            call(_l(**over))
        assert e.value.status == status and binding.came_last_error(None) != ""


@pytest.mark.parametrize("call,over,status", [
    (FORWARD, dict(y=None), 1), (FORWARD, dict(mean=None), 1), (FORWARD, dict(rstd=None), 1), (FORWARD, dict(eps=-1.0), 5), (FORWARD, dict(eps=float("nan")), 5),
    (FORWARD, dict(eps=1e39), 5), (FORWARD, dict(flags=1), 11), (FORWARD, dict(y=0x100000), 12), (FORWARD, dict(y=0x1FFFF0), 12),
    (FORWARD, dict(bias=0x300010), 12), (FORWARD, dict(mean=0x300000), 12), (FORWARD, dict(bias=0x210001), 4),
    (BACKWARD, dict(dy=None), 1), (BACKWARD, dict(mean=None), 1), (BACKWARD, dict(dx_ld=7), 2), (BACKWARD, dict(dx_dtype=3), 3), (BACKWARD, dict(dx=0x400000), 12),
    (BACKWARD, dict(dweight=0x610000), 12), (BACKWARD, dict(dbias=0x200000), 12), (BACKWARD, dict(dx=0x500002), 4), (BACKWARD, dict(dbias=0x610001), 4),
    (BACKWARD, dict(dx=0x700000), 12),
])
def test_refused_in_one_direction(call, over, status):
    with pytest.raises(binding.CameError) as e:
        call(_l(**over))
    assert e.value.status == status


def test_workspace():
    L = binding.load()
    assert L.came_layernorm_workspace(_l(), None) == 1 and L.came_layernorm_forward(None, 0, None) == 1
    size = binding.came_layernorm_workspace(_l(rows=1000, cols=256, x_ld=256, y_ld=256, dx_ld=256))
    assert size >= 2 * 4 * 256
    assert binding.came_layernorm_workspace(_l(dweight=None, dbias=None)) <= 256
    with pytest.raises(binding.CameError) as e:
        binding.came_layernorm_backward(_l(), None, 1 << 20)
    assert e.value.status == 1
    with pytest.raises(binding.CameError) as e:
        binding.came_layernorm_backward(_l(), 0x800008, 1 << 20)
    assert e.value.status == 4
    with pytest.raises(binding.CameError) as e:
        binding.came_layernorm_backward(_l(), 0x800000, 16)
    assert e.value.status == 2


def test_without_gpu_reports_device_error():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in (FORWARD, BACKWARD):
        for over in ({}, dict(rows=0, x=None, y=None, dy=None, dx=None, mean=None, rstd=None)):
            with pytest.raises(binding.CameError) as e:
                call(_l(**over))
            assert e.value.status == 7
