"""A small language model with one attention layer, trained with the operators that stand beside the lookup and the clipping.

    python examples/attention_lm.py [steps]

Tokens are looked up, normalised, mixed by causal attention whose scores get a learned bias for the distance of query
and key, normalised again, and compared with the table (tied).  Layer norm, bias and lookup are this library's, as parts
of autograd's graph; ``GradClip`` reads all gradients once, and ``AdamWOptimizer`` takes the clipping coefficient from
device memory.  The matrices' states have 8 bits, the vectors' and the bias table's 32."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.tied_lm import batches  # noqa: E402
from paper_2307_02047_b200 import binding  # noqa: E402


class AttentionLM:
    def __init__(self, vocab=997, dim=128, heads=4, buckets=16, far=32, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda *s, std: torch.randn(*s, generator=gen, device=device) * std  # noqa: E731
        self.heads, self.far = heads, far
        self.params = {
            "table": new(vocab, dim, std=0.02), "qkv": new(dim, 3 * dim, std=dim ** -0.5), "out": new(dim, dim, std=dim ** -0.5),
            "bias": new(buckets, heads, std=0.1), "norm1": torch.ones(dim, device=device), "shift1": torch.zeros(dim, device=device),
            "norm2": torch.ones(dim, device=device), "shift2": torch.zeros(dim, device=device)}
        for p in self.params.values():
            p.requires_grad_(True)

    def loss(self, ids, targets, lookup=binding.embed_forward, norm=binding.layer_norm, bias=binding.position_bias_forward):
        p, (batch, length) = self.params, ids.shape
        x = lookup(p["table"], ids, math.sqrt(p["table"].shape[1]))
        q, k, v = (norm(x, p["norm1"], p["shift1"]) @ p["qkv"]).view(batch, length, 3, self.heads, -1).permute(2, 0, 3, 1, 4)
        scores = q @ k.transpose(-1, -2) * q.shape[-1] ** -0.5 + bias(p["bias"], length, length, bidirectional=False, max_distance=self.far)
        scores = scores.masked_fill(torch.ones(length, length, dtype=torch.bool, device=ids.device).triu(1), float("-inf"))
        x = x + (torch.softmax(scores, -1) @ v).transpose(1, 2).reshape(batch, length, -1) @ p["out"]
        logits = norm(x, p["norm2"], p["shift2"]) @ p["table"].t()
        return torch.nn.functional.cross_entropy(logits.flatten(0, -2), targets.flatten(), ignore_index=-1)


def train(steps=300, vocab=997, dim=128, batch=32, length=64, max_norm=1.0, lr=3e-3, seed=0, report=None):
    """Losses and gradient norms of every step."""
    model = AttentionLM(vocab, dim, seed=seed)
    params = list(model.params.values())
    grads = [torch.zeros_like(p) for p in params]
    for p, g in zip(params, grads):
        p.grad = g                                       # autograd adds in place
    clip = binding.GradClip(grads)
    opt = binding.AdamWOptimizer([p.detach() for p in params], grads, state_bits=[8 if p.shape[0] > 64 and p.dim() == 2 else 32 for p in params],
                                 flags=[0 if p.dim() == 2 else binding.CAME_T_NO_WEIGHT_DECAY for p in params], seed=seed)
    data, losses, norms = batches(vocab, batch, length, seed + 1), [], []
    for step in range(1, steps + 1):
        ids, targets = next(data)
        for g in grads:
            g.zero_()
        loss = model.loss(ids, targets)
        loss.backward()
        total_norm, coef, _ = clip.norm(max_norm)
        opt.step(binding.came_lr_warmup(lr, 0.0, step, 20), weight_decay=0.01, device_scale=coef)
        losses.append(loss.detach())
        norms.append(total_norm.clone())
        if report and step % 50 == 0:
            report(f"step {step}: loss {float(losses[-1]):.3f}, gradient norm {float(total_norm):.3f}")
    opt.close()
    clip.close()
    return torch.stack(losses), torch.stack(norms)


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 300, report=print)
