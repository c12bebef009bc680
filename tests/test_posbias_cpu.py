"""The buckets against whole-number arithmetic, and the refusals that are decided before any CUDA call."""
import random

import pytest

from paper_2307_02047_b200 import binding


def bucket(relative, buckets, far, both):
    """The definition in whole numbers: the largest step k with near (far / near)^(k / steps) <= d."""
    n = buckets // 2 if both else buckets
    near, steps = n // 2, n - n // 2
    d = abs(relative) if both else max(-relative, 0)
    if d >= near:
        k = 0
        while k < steps - 1 and far ** (k + 1) * near ** (steps - k - 1) <= d ** steps:
            k += 1
        d = near + k
    return d + (n if both and relative > 0 else 0)


def _p(**over):
    d = dict(table=0x10000, data=0x100000, device_offset=None, offset=0, q_len=5, k_len=7, batch=2, table_ld=4, batch_stride=140, head_stride=35, q_stride=7,
             heads=4, buckets=32, max_distance=128, table_dtype=0, data_dtype=0, flags=1)
    d.update(over)
    return binding.came_posbias(**d)


@pytest.mark.parametrize("buckets,far,both", [(32, 128, True), (32, 128, False), (8, 64, True), (4, 2, True), (4, 16, False), (2, 2, False), (64, 1024, False),
                                              (6, 9, True), (33, 17, False), (1024, 4096, True), (32, 9, True), (16, 1 << 20, False), (128, 100_000, True)])
def test_buckets(buckets, far, both):
    p = _p(buckets=buckets, max_distance=far, flags=int(both))
    rng = random.Random(buckets + far)
    near = set(range(-700, 701)) | {s * (far + d) for s in (1, -1) for d in (-1, 0, 1)} | {rng.randrange(-2 * far, 2 * far) for _ in range(200)}
    # powers at which a border is a whole number
    near |= {s * v + d for s in (1, -1) for v in (2 ** k for k in range(1, 21)) for d in (-1, 0, 1)}
    for r in sorted(near):
        assert binding.came_posbias_bucket(p, r) == bucket(r, buckets, far, both), r
    assert binding.came_posbias_bucket(p, -(1 << 62)) == bucket(-far, buckets, far, both)


FORWARD, BACKWARD = (lambda p: binding.came_posbias_forward(p)), (lambda p: binding.came_posbias_backward(p, 0x800000, 1 << 20))


@pytest.mark.parametrize("over,status", [
    (dict(q_len=-1), 2), (dict(k_len=(1 << 30) + 1), 2), (dict(heads=0), 2), (dict(heads=65536), 2), (dict(buckets=1, flags=0), 2), (dict(buckets=5), 2),
    (dict(buckets=2), 2), (dict(buckets=1026), 2), (dict(max_distance=8), 5), (dict(max_distance=(1 << 29) + 1), 5), (dict(offset=(1 << 40) + 1), 2),
    (dict(table_ld=3), 2), (dict(table_dtype=2), 3), (dict(data_dtype=-1), 3), (dict(flags=5), 11), (dict(table=None), 1), (dict(data=None), 1),
    (dict(table=0x10002), 4), (dict(data=0x100001), 4), (dict(device_offset=0x20004), 4), (dict(data=0x10010), 12), (dict(q_len=1 << 30, k_len=1 << 30), 2),
])
def test_refused_in_both_directions(over, status):
    for call in (FORWARD, BACKWARD):
        with pytest.raises(binding.CameError) as e:
            call(_p(**over))
        assert e.value.status == status and binding.came_last_error(None) != ""


@pytest.mark.parametrize("call,over,status", [
    (FORWARD, dict(flags=3), 11), (FORWARD, dict(device_offset=0x100008), 12), (BACKWARD, dict(device_offset=0x10008), 12), (BACKWARD, dict(batch=-1), 2),
    (BACKWARD, dict(q_stride=-1), 2), (BACKWARD, dict(batch_stride=1 << 60), 2),
])
def test_refused_in_one_direction(call, over, status):
    with pytest.raises(binding.CameError) as e:
        call(_p(**over))
    assert e.value.status == status


def test_workspace_and_null():
    L = binding.load()
    assert L.came_posbias_workspace(_p(), None) == 1 and L.came_posbias_forward(None, 0, None) == 1 and L.came_posbias_bucket(None, 0, None) == 1
    assert binding.came_posbias_workspace(_p()) >= 4 * 32 * 4
    for ws, size, status in ((None, 1 << 20, 1), (0x800008, 1 << 20, 4), (0x800000, 16, 2)):
        with pytest.raises(binding.CameError) as e:
            binding.came_posbias_backward(_p(), ws, size)
        assert e.value.status == status


def test_without_gpu_reports_device_error():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for call in (FORWARD, BACKWARD):
        for over in ({}, dict(q_len=0, data=None)):
            with pytest.raises(binding.CameError) as e:
                call(_p(**over))
            assert e.value.status == 7


@pytest.mark.parametrize("heads,q,k", [(1, 1, 1), (64, 1, 5), (4, 65, 63), (2, 301, 303)])
def test_workspace_of_batches_at_odd_strides(heads, q, k):
    """Batches begin at one of eight places: eight times the sums at most of batches that all begin at one."""
    for batch in (1, 5, 100, 1 << 20):
        sizes = [binding.came_posbias_workspace(_p(heads=heads, table_ld=heads, q_len=q, k_len=k, q_stride=k, head_stride=q * k, batch=batch, table=1 << 50,
                                                   batch_stride=stride)) for stride in (-(-heads * q * k // 8) * 8, -(-heads * q * k // 8) * 8 + 1)]
        assert sizes[1] <= 8 * sizes[0]
