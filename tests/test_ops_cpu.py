"""Refusals of the gradient-norm entry points that are decided before any CUDA call."""
import ctypes

import pytest

from paper_2307_02047_b200 import binding


def _clip(grad=0x10000, out=None, numel=64, gdt=0, odt=0):
    return binding.came_clip_tensor(grad, out, numel, gdt, odt)


@pytest.mark.parametrize("descs,status", [
    ([_clip(numel=-1)], 2), ([_clip(numel=(1 << 40) + 1)], 2), ([_clip(gdt=2)], 3), ([_clip(out=0x20000, odt=9)], 3),
    ([_clip(grad=None)], 1), ([_clip(grad=0x10002)], 4), ([_clip(grad=0x10001, gdt=1)], 4), ([_clip(out=0x20001, odt=1)], 4),
    ([_clip(out=0x20000), _clip(grad=0x30000)], 1),                       # one has an output, the other none
    ([_clip(out=0x10080)], 12),                                           # output inside its own gradient
    ([_clip(out=0x10000, odt=1)], 12),                                    # in place, but another type
    ([_clip(out=0x20000), _clip(grad=0x20080, out=0x40000)], 12),         # output over another's gradient
    ([_clip(out=0x20000), _clip(grad=0x30000, out=0x20000)], 12),         # the same output twice
])
def test_clip_create_refuses(descs, status):
    with pytest.raises(binding.CameError) as e:
        binding.came_clip_create(descs)
    assert e.value.status == status and binding.came_last_error(None) != ""


def test_clip_null_arguments():
    L = binding.load()
    ctx = ctypes.c_void_p()
    arr = (binding.came_clip_tensor * 1)(_clip())
    assert L.came_clip_create(None, arr, 1, 0) == 1
    assert L.came_clip_create(ctypes.byref(ctx), None, 1, 0) == 1
    assert L.came_clip_create(ctypes.byref(ctx), arr, 0, 0) == 2
    assert ctx.value is None
    assert L.came_clip_norm(None, binding.came_clip_params(1.0, 0.0, 1.0), None, 0x1000, None) == 1
    assert L.came_clip_grads(None, None, None, None, None) == 1
    assert L.came_clip_destroy(None) == 1
    assert L.came_step_scaled(None, None, None, None, None) == 1


def test_operators_without_gpu_report_device_error():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for descs in ([_clip()], [_clip(numel=0, grad=None)], [_clip(out=0x10000)]):
        with pytest.raises(binding.CameError) as e:
            binding.came_clip_create(descs)
        assert e.value.status == 7      # CAME_ERR_DEVICE: no silent CPU fallback
