"""Refusals of the AdamW entry points that are decided before any CUDA call."""
import ctypes

import pytest

from paper_2307_02047_b200 import binding


def _t(**over):
    d = dict(param=0x10000, grad=0x20000, m=0x30000, v=0x40000, m_scale=None, v_scale=None, param_bf16=None, numel=64, grad_dtype=0,
             state_bits=32, flags=0, reserved=0)
    d.update(over)
    return binding.came_adamw_tensor(**d)


@pytest.mark.parametrize("descs,status", [
    ([_t(numel=-1)], 2), ([_t(numel=(1 << 39) + 1)], 2), ([_t(grad_dtype=2)], 3), ([_t(state_bits=16)], 3), ([_t(flags=2)], 11), ([_t(reserved=1)], 2),
    ([_t(param=None)], 1), ([_t(grad=None)], 1), ([_t(m=None)], 1), ([_t(v=None)], 1), ([_t(state_bits=8)], 1), ([_t(state_bits=8, m_scale=0x50000)], 1),
    ([_t(param=0x10002)], 4), ([_t(grad=0x20002)], 4), ([_t(grad=0x20001, grad_dtype=1)], 4), ([_t(m=0x30001)], 4), ([_t(param_bf16=0x50001)], 4),
    ([_t(m=0x10080)], 12), ([_t(v=0x30000)], 12), ([_t(grad=0x100FC)], 12), ([_t(param_bf16=0x200F0)], 12),
    ([_t(state_bits=8, m_scale=0x50000, v_scale=0x50000)], 12), ([_t(), _t(grad=0x60000)], 12),
    ([_t(), _t(param=0x110000, m=0x130000, v=0x140000, grad=0x10000)], 12),
])
def test_create_refuses(descs, status):
    with pytest.raises(binding.CameError) as e:
        binding.came_adamw_create(descs)
    assert e.value.status == status and binding.came_last_error(None) != ""


def test_gradients_may_be_shared():
    """Two tensors may read one gradient: what follows is the missing GPU here, or a context."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for descs in ([_t(), _t(param=0x110000, m=0x130000, v=0x140000)], [_t(numel=0, param=None, grad=None, m=None, v=None)]):
        with pytest.raises(binding.CameError) as e:
            binding.came_adamw_create(descs)
        assert e.value.status == 7


def test_null_arguments_and_counts():
    L = binding.load()
    ctx = ctypes.c_void_p()
    arr = (binding.came_adamw_tensor * 1)(_t())
    assert L.came_adamw_create(None, arr, 1, 0, 0) == 1
    assert L.came_adamw_create(ctypes.byref(ctx), None, 1, 0, 0) == 1
    assert L.came_adamw_create(ctypes.byref(ctx), arr, 0, 0, 0) == 2
    assert L.came_adamw_create(ctypes.byref(ctx), arr, 1, 0, 2) == 11
    assert ctx.value is None
    assert L.came_adamw_step(None, binding.came_adamw_hparams(), None, None, None, None) == 1
    assert L.came_adamw_destroy(None) == 1
