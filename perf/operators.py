"""What is measured of the operators that stand around the optimizer step: the global gradient
norm, clipping, the embedding lookup and its gradient.

``run`` computes a case either in plain elementary torch operations (``own`` false) or through
this repository's entry points (``own`` true); ``exact`` gives the same results in 64 bits.

    norm    n_i = s sqrt(sum g_i^2),  N = sqrt(sum n_i^2),
            coef = 1 if N + eps <= max_norm else max_norm / (N + eps)
    clip    the same, and out_i = g_i * s * coef
    lookup  out[t] = scale * W[id_t], zero where id_t is not a row of W
    grad    dW[v] = scale * sum over the tokens t with id_t = v of dY[t]; ``add``: added to dW
"""
import math

import torch

own = False

EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
IT = {"i32": torch.int32, "i64": torch.int64}
ALIGN = 8          # elements: where the next tensor of a flat gradient buffer may start


# ---- the parameter sets whose gradients are measured ------------------------------------------

def _bert_like(hidden, ffn, layers, vocab, pos):
    shapes = [vocab * hidden, pos * hidden]
    per = [hidden * hidden] * 4 + [hidden * ffn] * 2 + [hidden] * 4 + [ffn, hidden] + [hidden] * 4
    return shapes + per * layers


def _gpt2_like(hidden, ffn, layers, vocab, pos):
    per = [3 * hidden * hidden, hidden * hidden, hidden * ffn, hidden * ffn, 3 * hidden, hidden, ffn, hidden] + [hidden] * 4
    return [vocab * hidden, pos * hidden] + per * layers


def _llama_like(hidden, ffn, layers, vocab):
    per = [hidden * hidden] * 4 + [hidden * ffn] * 3 + [hidden] * 2
    return [vocab * hidden] + per * layers + [hidden, vocab * hidden]


def _sizes(case):
    """Lengths of the tensors of a norm or clip case."""
    kind = case["set"]
    if kind == "toy":
        return [512 * 256, 256]
    if kind == "ragged":
        return [513 * 1030, 1001, 33 * 65, 1, 7, 300]
    if kind == "bert_base":
        return _bert_like(768, 3072, 12, 30522, 512)
    if kind == "gpt2_medium":
        return _gpt2_like(1024, 4096, 24, 50257, 1024)
    if kind == "llama7b":
        return _llama_like(4096, 11008, 32, 32000)
    # "drawn": `count` tensors from 1 to `most` elements, spread over the logarithm
    g = torch.Generator().manual_seed(case["shapes"])
    u = torch.rand(case["count"], generator=g, dtype=torch.float64)
    return [max(1, int(x)) for x in torch.exp(u * math.log(case["most"])).tolist()]


def listed():
    return [
        # the smallest set anyone steps: one matrix and its bias, where the call itself counts
        {"name": "norm toy f32", "op": "norm", "set": "toy", "dtype": "f32", "max_norm": 0.1},
        # 194 tensors of a BERT-base-shaped model, fp32 gradients
        {"name": "norm bert-base f32", "op": "norm", "set": "bert_base", "dtype": "f32", "max_norm": 1.0},
        # 291 tensors of a LLaMA-7B-shaped model, bf16 gradients: 13.5 GB
        {"name": "norm llama-7b bf16", "op": "norm", "set": "llama7b", "dtype": "bf16", "max_norm": 1.0},
        # a few tensors of odd lengths, one of a single element
        {"name": "clip ragged f32", "op": "clip", "set": "ragged", "dtype": "f32", "out": "f32", "max_norm": 0.1},
        # 290 tensors of a GPT-2-medium-shaped model, clipped into the buffer that the step reads
        {"name": "clip gpt2-medium bf16", "op": "clip", "set": "gpt2_medium", "dtype": "bf16", "out": "bf16", "max_norm": 1.0},
        # one token for each of eight sequences
        {"name": "lookup 8 tokens bf16", "op": "lookup", "tokens": 8, "rows": 32000, "cols": 4096, "dtype": "bf16", "out": "bf16",
         "ids": "i64", "scale": 1.0, "holes": 0.0},
        # a training batch of 16 x 1024 tokens; fp32 parameters, bf16 activations, scaled
        {"name": "lookup gpt2-medium f32", "op": "lookup", "tokens": 16384, "rows": 50257, "cols": 1024, "dtype": "f32", "out": "bf16",
         "ids": "i64", "scale": 32.0, "holes": 0.0},
        # a large batch, 32 x 4096 tokens, a tenth of them padding
        {"name": "lookup 128k tokens bf16", "op": "lookup", "tokens": 131072, "rows": 128256, "cols": 4096, "dtype": "bf16", "out": "bf16",
         "ids": "i32", "scale": 1.0, "holes": 0.1},
        # the smallest: a few tokens, an odd number of them, in a small table
        {"name": "grad toy f32", "op": "grad", "tokens": 33, "rows": 512, "cols": 256, "dtype": "f32", "out": "f32",
         "ids": "i64", "scale": 1.0, "holes": 0.0, "add": False},
        # the gradient of the 16 x 1024 batch
        {"name": "grad gpt2-medium bf16", "op": "grad", "tokens": 16384, "rows": 50257, "cols": 1024, "dtype": "bf16", "out": "bf16",
         "ids": "i64", "scale": 32.0, "holes": 0.0, "add": False},
        # a large batch against a small vocabulary: most rows have tokens, some have thousands
        {"name": "grad llama-7b bf16", "op": "grad", "tokens": 131072, "rows": 32000, "cols": 4096, "dtype": "bf16", "out": "bf16",
         "ids": "i32", "scale": 1.0, "holes": 0.05, "add": False},
        # a table tied to the output head: added to the head's gradient, a sixth of the tokens padding
        {"name": "grad tied bert-base f32", "op": "grad", "tokens": 8192, "rows": 30522, "cols": 768, "dtype": "f32", "out": "f32",
         "ids": "i64", "scale": 1.0, "holes": 0.15, "add": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "clip", "lookup", "grad", "grad"])
    dtype, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    if op in ("norm", "clip"):
        count = _log(rng, 1, 300)
        case = {"op": op, "set": "drawn", "shapes": rng.randrange(1 << 30), "count": count, "most": _log(rng, 1000, 30_000_000),
                "dtype": dtype, "max_norm": round(math.exp(rng.uniform(math.log(0.01), math.log(10.0))), 4)}
        if op == "clip":
            case["out"] = out
        return case
    cols = _log(rng, 64, 8192)
    cols = cols if rng.random() < 0.3 else max(64, cols // 64 * 64)       # mostly what models have, odd ones among them
    rows = _log(rng, 100, min(150_000, (1 << 29) // cols))
    tokens = _log(rng, 1, min(131_072, (1 << 29) // cols))
    case = {"op": op, "tokens": tokens, "rows": rows, "cols": cols, "dtype": dtype, "out": out, "ids": rng.choice(["i32", "i64"]),
            "scale": rng.choice([1.0, round(math.sqrt(cols), 3)]), "holes": rng.choice([0.0, 0.0, 0.1, 0.5]) if tokens >= 32 else 0.0}
    if op == "grad":
        case["add"] = rng.random() < 0.3
    return case


# ---- inputs -------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _gradients(case, seed):
    """The gradients as views of one flat buffer, each with a spread of its own."""
    sizes, gen = _sizes(case), _generator(seed)
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // ALIGN) * ALIGN
    flat = torch.zeros(total, dtype=DT[case["dtype"]], device="cuda")
    views = [flat[a:a + n] for a, n in zip(starts, sizes)]
    sigma = torch.exp(torch.rand(len(sizes), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * math.log(1e3)) * 1e-5
    for v, s in zip(views, sigma.tolist()):          # one spread for a tensor: log-uniform in [1e-5, 1e-2]
        v.normal_(0.0, s, generator=gen)
    return flat, views


def _tokens(case, seed):
    """Token ids whose frequency falls as 1/rank, low ids first as in merged vocabularies; `holes` of them are padding (-1)."""
    gen = _generator(seed)
    n, rows = case["tokens"], case["rows"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(rows + 1)) - 1).to(torch.int64).clamp_(0, rows - 1)
    hole = torch.rand(n, generator=gen, device="cuda") < case["holes"]
    return torch.where(hole, -1, ids).to(IT[case["ids"]]), gen


def prepare(case, seed):
    s = {"case": case}
    if case["op"] in ("norm", "clip"):
        s["flat"], s["grads"] = _gradients(case, seed)
        if case["op"] == "clip":
            s["out_flat"] = torch.zeros(s["flat"].shape, dtype=DT[case["out"]], device="cuda")
            a = s["flat"].data_ptr()
            at = [(g.data_ptr() - a) // g.element_size() for g in s["grads"]]
            s["outs"] = [s["out_flat"][k:k + g.numel()] for k, g in zip(at, s["grads"])]
        if own:
            from paper_2307_02047_b200 import binding
            s["clip"] = binding.GradClip(s["grads"], s.get("outs"))
        return s
    s["ids"], gen = _tokens(case, seed)
    if case["op"] == "lookup":
        s["table"] = torch.empty(case["rows"], case["cols"], dtype=DT[case["dtype"]], device="cuda").normal_(0.0, 0.02, generator=gen)
    else:
        s["dy"] = torch.empty(case["tokens"], case["cols"], dtype=DT[case["dtype"]], device="cuda").normal_(0.0, 1e-3, generator=gen)
        s["grad"] = torch.empty(case["rows"], case["cols"], dtype=DT[case["out"]], device="cuda")
        if case["add"]:
            s["grad"].normal_(0.0, 1e-3, generator=gen)
    return s


# ---- one pass -----------------------------------------------------------------------------------

def _plain_norm(grads, max_norm):
    sums = torch.stack([g.float().square().sum() for g in grads])
    total = sums.sum().sqrt()
    coef = torch.where(total + EPS <= max_norm, 1.0, max_norm / (total + EPS))
    return total, coef, sums.sqrt()


def _plain_lookup(table, ids, scale, dtype):
    ids = ids.long()
    row = (ids >= 0) & (ids < table.shape[0])
    x = table[torch.where(row, ids, 0)].float() * scale
    return torch.where(row[:, None], x, 0.0).to(dtype)


def _plain_grad(dy, ids, grad, scale, add):
    ids = ids.long()
    row = (ids >= 0) & (ids < grad.shape[0])
    x = torch.where(row[:, None], dy.float() * scale, 0.0)
    total = grad.float() if add else torch.zeros_like(grad, dtype=torch.float32) if grad.dtype != torch.float32 else grad.zero_()
    total.index_add_(0, torch.where(row, ids, 0), x)
    if total is not grad:
        grad.copy_(total)
    return grad


def run(state):
    c = state["case"]
    if own:
        from paper_2307_02047_b200 import binding
        if c["op"] == "norm":
            return state["clip"].norm(c["max_norm"], EPS)
        if c["op"] == "clip":
            return *state["clip"].clip(c["max_norm"], EPS), state["out_flat"]
        if c["op"] == "lookup":
            return binding.embed_forward(state["table"], state["ids"], c["scale"], out_dtype=DT[c["out"]])
        return binding.embed_backward(state["dy"], state["ids"], state["grad"], c["scale"], accumulate=c["add"])
    if c["op"] in ("norm", "clip"):
        total, coef, each = _plain_norm(state["grads"], c["max_norm"])
        if c["op"] == "norm":
            return total, coef, each
        state["out_flat"].copy_(state["flat"].float() * coef)
        return total, coef, each, state["out_flat"]
    if c["op"] == "lookup":
        return _plain_lookup(state["table"], state["ids"], c["scale"], DT[c["out"]])
    return _plain_grad(state["dy"], state["ids"], state["grad"], c["scale"], c["add"])


# ---- what a pass cannot do without ---------------------------------------------------------------

def _distinct(case):
    """Expected number of distinct rows among the tokens that are not padding."""
    n = case["tokens"] * (1.0 - case["holes"])
    r = torch.arange(1, case["rows"] + 1, dtype=torch.float64)
    p = (torch.log1p(1.0 / r)) / math.log(case["rows"] + 1)
    return float((1.0 - torch.exp(n * torch.log1p(-p))).sum()) if case["rows"] > 1 else min(1.0, n)


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    if case["op"] in ("norm", "clip"):
        n = sum(_sizes(case))
        b = n * size[case["dtype"]]
        return {"bytes": b, "flops": 2 * n} if case["op"] == "norm" else {"bytes": b + n * size[case["out"]], "flops": 3 * n}
    t, cols, seen = case["tokens"], case["cols"], _distinct(case)
    valid = t * (1.0 - case["holes"])
    if case["op"] == "lookup":
        return {"bytes": seen * cols * size[case["dtype"]] + t * cols * size[case["out"]] + t * size[case["ids"]], "flops": t * cols}
    written = 2 * seen if case["add"] else case["rows"]
    return {"bytes": valid * cols * size[case["dtype"]] + written * cols * size[case["out"]] + t * size[case["ids"]], "flops": valid * cols}


# ---- in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] in ("norm", "clip"):
        flat, grads = _gradients(case, seed)
        squares = []
        for g in grads:
            parts = [torch.linalg.vector_norm(p, dtype=torch.float64).item() for p in g.split(1 << 27)]
            squares.append(math.fsum(x * x for x in parts))
        norm = math.sqrt(math.fsum(squares))
        coef = min(1.0, case["max_norm"] / (norm + EPS))
        got = [torch.tensor(norm, dtype=torch.float64), torch.tensor(coef, dtype=torch.float64), torch.tensor(squares, dtype=torch.float64).sqrt()]
        return got if case["op"] == "norm" else got + [flat.double() * coef]
    ids, gen = _tokens(case, seed)
    ids = ids.long()
    kept = ((ids >= 0) & (ids < case["rows"])).nonzero()[:, 0]
    if case["op"] == "lookup":
        table = torch.empty(case["rows"], case["cols"], dtype=DT[case["dtype"]], device="cuda").normal_(0.0, 0.02, generator=gen)
        out = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
        out[kept] = table.double()[ids[kept]] * case["scale"]
        return out
    dy = torch.empty(case["tokens"], case["cols"], dtype=DT[case["dtype"]], device="cuda").normal_(0.0, 1e-3, generator=gen)
    grad = torch.empty(case["rows"], case["cols"], dtype=DT[case["out"]], device="cuda")
    if case["add"]:
        grad.normal_(0.0, 1e-3, generator=gen)
    # by columns: the tokens of a row side by side, summed as differences of a running total
    order = kept[torch.argsort(ids[kept], stable=True)]
    count = torch.bincount(ids[kept], minlength=case["rows"])
    last = torch.cumsum(count, 0)
    out = grad.double() if case["add"] else torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // max(1, case["tokens"]))
    for a in range(0, case["cols"], step):
        run_ = torch.cumsum(dy[order, a:a + step].double(), 0)
        run_ = torch.cat([torch.zeros_like(run_[:1]) if len(run_) else torch.zeros(1, min(step, case["cols"] - a), dtype=torch.float64, device="cuda"), run_])
        out[:, a:a + step] += case["scale"] * (run_[last] - run_[last - count])
    return out
