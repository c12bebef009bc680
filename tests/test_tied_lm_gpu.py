"""The example that runs the lookup, its gradient, the norm and the clipped step together."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_gradients_equal_autograd():
    """The tied table's gradient (head by autograd, lookup added by the kernel) against torch's own
    indexing.  fp32 sums of at most a few thousand terms on both sides: 1e-5 of the largest element."""
    import torch
    from examples import tied_lm
    torch.manual_seed(0)
    model = tied_lm.TiedLM(vocab=211, dim=72)
    ids, targets = next(tied_lm.batches(211, 16, 40, 3))
    model.loss(ids, targets).backward()
    got = [g.clone() for g in model.grads]
    table, mix, bias = (p.detach().double().requires_grad_() for p in model.params)
    x = table[ids.clamp(min=0)] * (ids >= 0)[..., None] * model.scale
    logits = torch.tanh(x @ mix + bias) @ table.t()
    torch.nn.functional.cross_entropy(logits.flatten(0, -2), targets.flatten(), ignore_index=-1).backward()
    for a, b in zip(got, (table.grad, mix.grad, bias.grad)):
        assert float((a.double() - b).abs().max()) <= 1e-5 * float(b.abs().max())


def test_training_lowers_the_loss_and_is_reproducible_around_torch():
    import torch
    from examples import tied_lm
    losses, norms = tied_lm.train(steps=200, vocab=301, dim=64)
    assert bool(losses.isfinite().all()) and bool(norms.isfinite().all())
    assert abs(float(losses[0]) - math.log(301)) < 1.0
    assert float(losses[-20:].mean()) < float(losses[0]) - 1.5
