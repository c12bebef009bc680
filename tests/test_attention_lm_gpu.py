"""The example that runs layer norm, position bias, lookup, clipping and AdamW together."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_gradients_equal_autograd():
    """Against torch's own indexing and elementary operations, both in fp32: every gradient is a sum of at most 4 x 24 x 101 terms through
    a few products of 32 to 96 terms; 256 roundings of 2^-24 in a row, 1.5e-5, of the largest gradient of the tensor hold that."""
    import torch
    from examples.attention_lm import AttentionLM, batches
    from tests.test_posbias_cpu import bucket
    model = AttentionLM(101, 32, heads=2, buckets=8, far=12, seed=1)
    ids, targets = next(batches(101, 4, 24, 2))
    model.loss(ids, targets).backward()
    got = {k: p.grad.clone() for k, p in model.params.items()}

    def lookup(table, ids, scale):
        return torch.where((ids >= 0)[..., None], table[ids.clamp(min=0)] * scale, 0.0)

    def norm(x, w, b):
        d = x - x.mean(-1, keepdim=True)
        return d * torch.rsqrt((d * d).mean(-1, keepdim=True) + 1e-5) * w + b

    def bias(table, q, k, bidirectional, max_distance):
        where = torch.tensor([[bucket(j - i, table.shape[0], max_distance, bidirectional) for j in range(k)] for i in range(q)], device="cuda")
        return table[where].permute(2, 0, 1)
    for p in model.params.values():
        p.grad = None
    model.loss(ids, targets, lookup, norm, bias).backward()
    for name, p in model.params.items():
        assert float((got[name] - p.grad).abs().max()) <= 1.5e-5 * float(p.grad.abs().max()), name


def test_steps_run_and_repeat():
    """Finite losses and norms; a second run gives the same bits up to the library products of torch."""
    import torch
    from examples import attention_lm
    losses, norms = attention_lm.train(steps=4, vocab=101, dim=64, batch=4, length=16)
    assert bool(losses.isfinite().all()) and bool((norms > 0).all()) and losses.shape == norms.shape == (4,)
    assert abs(float(losses[0]) - math.log(101)) < 1.5           # (near a uniform guess before the first step)
    again, _ = attention_lm.train(steps=4, vocab=101, dim=64, batch=4, length=16)
    assert torch.allclose(losses, again, rtol=1e-4, atol=0)
