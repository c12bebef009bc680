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


def _embed(**over):
    d = dict(table=0x10000, data=0x20000, ids=0x30000, rows=10, cols=8, tokens=4, table_ld=8, data_ld=8, padding_row=0,
             scale=1.0, table_dtype=0, data_dtype=0, id_dtype=1, flags=0, reserved=0)
    d.update(over)
    return binding.came_embed(**d)


@pytest.mark.parametrize("over,status", [
    (dict(rows=0), 2), (dict(cols=0), 2), (dict(tokens=-1), 2), (dict(rows=(1 << 31) - 1), 2), (dict(tokens=1 << 31), 2),
    (dict(table_ld=7), 2), (dict(data_ld=7), 2), (dict(table_ld=1 << 40), 2), (dict(table_dtype=2), 3), (dict(data_dtype=-1), 3),
    (dict(id_dtype=2), 3), (dict(flags=8), 11), (dict(reserved=1), 2), (dict(scale=float("nan")), 5), (dict(table=None), 1),
    (dict(data=None), 1), (dict(ids=None), 1), (dict(table=0x10002), 4), (dict(data=0x20001), 4), (dict(ids=0x30004), 4),
    (dict(data=0x10010), 12),
])
def test_embed_refuses_before_any_cuda_call(over, status):
    for call in (binding.came_embed_workspace, lambda e: binding.came_embed_forward(e), lambda e: binding.came_embed_backward(e, 0x40000, 1 << 20)):
        with pytest.raises(binding.CameError) as e:
            call(_embed(**over))
        assert e.value.status == status and binding.came_last_error(None) != ""


def test_embed_workspace_and_flags():
    L = binding.load()
    assert L.came_embed_workspace(_embed(), None) == 1 and L.came_embed_forward(None, 0, None) == 1
    small, large = binding.came_embed_workspace(_embed(tokens=0, data=None, ids=None)), binding.came_embed_workspace(_embed(tokens=1000, data=0x100000))
    assert 0 < small < large
    with pytest.raises(binding.CameError) as e:
        binding.came_embed_forward(_embed(flags=1))          # the flags belong to the gradient
    assert e.value.status == 11
    with pytest.raises(binding.CameError) as e:
        binding.came_embed_forward(_embed(data=0x2FFF0))     # the output runs into the ids
    assert e.value.status == 12


def test_embed_without_gpu_reports_device_error():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in (lambda e: binding.came_embed_forward(e), lambda e: binding.came_embed_backward(e, 0x40000, 1 << 20)):
        with pytest.raises(binding.CameError) as e:
            call(_embed())
        assert e.value.status == 7


@pytest.mark.parametrize("scale", [1e39, -3.5e38, 1.7976931348623157e308, 1e-46, -1e-300, float("inf")])
def test_a_scale_that_fp32_does_not_hold_is_refused(scale):
    """The kernels multiply by the fp32 value: infinity would make NaN of zeros, and zero would drop the data."""
    for call in (binding.came_embed_workspace, lambda e: binding.came_embed_forward(e), lambda e: binding.came_embed_backward(e, 0x40000, 1 << 20)):
        with pytest.raises(binding.CameError) as e:
            call(_embed(scale=scale))
        assert e.value.status == binding.CAME_ERR_HPARAM


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-40, -1.5e-45, 3.4028234663852886e38, -3.4e38])
def test_a_scale_that_fp32_holds_is_taken(scale):
    assert binding.came_embed_workspace(_embed(scale=scale)) > 0
