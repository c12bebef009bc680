"""A small tied-embedding language model trained with everything this library has around the step.

    python examples/tied_lm.py [steps]

The table is looked up (scaled), mixed by one hidden matrix and used again as the output head.
Its gradient has two parts: autograd adds the head's, and the lookup's is added to the same buffer
by ``embed_backward(accumulate=True)``.  ``GradClip`` then reads all gradients once, and
``CameOptimizer.step`` takes the clipping coefficient from device memory: no pass writes clipped
gradients, and the host never waits for the norm.  The data is a random Markov chain over the
vocabulary, with padding (id -1) at the end of some rows."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2307_02047_b200 import binding  # noqa: E402


class Lookup(torch.autograd.Function):
    """scale * table[ids]; its backward adds to the table's gradient buffer itself."""

    @staticmethod
    def forward(ctx, anchor, table, grad, ids, scale):
        ctx.save_for_backward(ids)
        ctx.grad, ctx.scale = grad, scale
        return binding.embed_forward(table, ids, scale)

    @staticmethod
    def backward(ctx, dy):
        (ids,) = ctx.saved_tensors
        binding.embed_backward(dy.contiguous(), ids, ctx.grad, ctx.scale, accumulate=True)
        return None, None, None, None, None


class TiedLM:
    def __init__(self, vocab=997, dim=128, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s, std: torch.randn(*s, generator=gen, device=device) * std  # noqa: E731
        self.params = [new(vocab, dim, std=0.02), new(dim, dim, std=dim ** -0.5), torch.zeros(dim, device=device)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        for p, g in zip(self.params, self.grads):
            p.requires_grad_(True)
            p.grad = g                                   # autograd adds in place
        self.anchor = torch.zeros((), device=device, requires_grad=True)     # makes the lookup part of the graph
        self.scale = math.sqrt(dim)

    def loss(self, ids, targets):
        table, mix, bias = self.params
        x = Lookup.apply(self.anchor, table.detach(), self.grads[0], ids, self.scale)
        h = torch.tanh(x @ mix + bias)
        logits = h @ table.t()
        return torch.nn.functional.cross_entropy(logits.flatten(0, -2), targets.flatten(), ignore_index=-1)


def batches(vocab, batch, length, seed, device="cuda"):
    """Rows of a Markov chain in which every token has three likely successors."""
    gen = torch.Generator(device=device).manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 3), generator=gen, device=device)
    while True:
        ids = torch.empty(batch, length + 1, dtype=torch.int64, device=device)
        ids[:, 0] = torch.randint(0, vocab, (batch,), generator=gen, device=device)
        pick = torch.randint(0, 3, (batch, length), generator=gen, device=device)
        for k in range(length):
            ids[:, k + 1] = successors[ids[:, k], pick[:, k]]
        cut = torch.randint(length // 2, length + 1, (batch,), generator=gen, device=device)
        pad = torch.arange(length, device=device)[None, :] >= cut[:, None]
        yield ids[:, :-1].masked_fill(pad, -1).contiguous(), ids[:, 1:].masked_fill(pad, -1).contiguous()


def train(steps=300, vocab=997, dim=128, batch=32, length=64, max_norm=1.0, lr=5e-3, seed=0, report=None):
    """Losses and gradient norms of every step."""
    model = TiedLM(vocab, dim, seed)
    clip = binding.GradClip(model.grads)
    opt = binding.CameOptimizer([p.detach() for p in model.params], model.grads)
    data, losses, norms = batches(vocab, batch, length, seed + 1), [], []
    for step in range(1, steps + 1):
        ids, targets = next(data)
        for g in model.grads:
            g.zero_()
        loss = model.loss(ids, targets)
        loss.backward()
        total_norm, coef, _ = clip.norm(max_norm)
        opt.step(device_scale=coef, lr=binding.came_lr_warmup(lr, 0.0, step, 20), beta1=0.9, beta2=0.999, beta3=0.9999,
                 eps1=1e-30, eps2=1e-16, clip_d=1.0)
        losses.append(loss.detach())
        norms.append(total_norm.clone())
        if report and step % 50 == 0:
            report(f"step {step}: loss {float(losses[-1]):.3f}, gradient norm {float(total_norm):.3f}")
    opt.close()
    clip.close()
    return torch.stack(losses), torch.stack(norms)


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 300, report=print)
