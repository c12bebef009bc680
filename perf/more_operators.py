"""What is measured of the operators that a training step has beside the optimizer step and the
embedding: an AdamW step over many tensors with states in 32 or 8 bits, layer norm with its backward
pass, and a learned relative position bias with its gradient.

``run`` computes a case either in plain elementary torch operations (``own`` false) or through
this repository's entry points (``own`` true); ``exact`` gives the same results in 64 bits.

    adamw   g = s * grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
            p -= lr (wd p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
            8 bits: after that m is stored as e4m3 and v as e5m2, with a power of two for each 256
            elements, rounded up or down at random: by 16 bits of a hash of (seed, t, element)
    ln      y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps), over the last dimension
    ln bwd  with h = (x - mean) rstd and d = dy w:  dx = rstd (d - mean(d) - h mean(d h)),
            dw = sum over rows of dy h,  db = sum over rows of dy;  ``add``: added to dw and db
    bias    out[h, i, j] = table[bucket(j - i - offset), h]
    bias grad   dtable[b, h] = sum over (batch, i, j) with that bucket of dout[., h, i, j];
            ``add``: added to dtable
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 256                                   # elements that share a scale in 8 bits
HP = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.1}
SEED = 0x5EED0123456789
STEPS_BEFORE = 1000                           # an optimizer in the middle of a run
LN_EPS = 1e-5


def listed():
    return [
        # the smallest set anyone steps: one matrix and its bias, where the call itself counts
        {"name": "adamw toy", "op": "adamw", "set": "toy", "dtype": "f32", "bits": 32, "copy": False},
        # 290 tensors of a GPT-2-medium-shaped model, everything in fp32
        {"name": "adamw gpt2-medium", "op": "adamw", "set": "gpt2_medium", "dtype": "f32", "bits": 32, "copy": False},
        # a few tensors of odd lengths, one of a single element: blocks that are not full
        {"name": "adamw ragged 8 bits", "op": "adamw", "set": "ragged", "dtype": "f32", "bits": 8, "copy": False},
        # bf16 gradients, 8-bit states, and the bf16 parameters that the next forward pass reads
        {"name": "adamw gpt2-medium 8 bits", "op": "adamw", "set": "gpt2_medium", "dtype": "bf16", "bits": 8, "copy": True},
        # one token for each of eight sequences
        {"name": "ln 8 tokens bf16", "op": "ln", "rows": 8, "cols": 4096, "dtype": "bf16", "out": "bf16", "weight": "bf16", "affine": "both"},
        # a training batch of 16 x 1024 tokens; fp32 parameters, bf16 activations
        {"name": "ln 16k tokens bf16", "op": "ln", "rows": 16384, "cols": 1024, "dtype": "bf16", "out": "bf16", "weight": "f32", "affine": "both"},
        # a small model in fp32: odd numbers of rows and columns, gradients added to what is there
        {"name": "ln bwd odd f32", "op": "ln bwd", "rows": 1001, "cols": 771, "dtype": "f32", "out": "f32", "weight": "f32", "affine": "both", "add": True},
        # a large batch, 32 x 4096 tokens
        {"name": "ln bwd 128k tokens bf16", "op": "ln bwd", "rows": 131072, "cols": 4096, "dtype": "bf16", "out": "bf16", "weight": "f32",
         "affine": "both", "add": False},
        # one token at the end of 2048 keys, looking back
        {"name": "bias one token", "op": "bias", "heads": 12, "q": 1, "k": 2048, "offset": 2047, "buckets": 32, "far": 128, "both": False,
         "dtype": "f32", "out": "bf16"},
        # 4096 x 4096 positions, looking both ways
        {"name": "bias 4096 bf16", "op": "bias", "heads": 16, "q": 4096, "k": 4096, "offset": 0, "buckets": 32, "far": 128, "both": True,
         "dtype": "f32", "out": "bf16"},
        # a batch of scores at the usual training length: summed over the batch too
        {"name": "bias grad batch bf16", "op": "bias grad", "batch": 16, "heads": 12, "q": 1024, "k": 1024, "offset": 0, "buckets": 32, "far": 128,
         "both": True, "dtype": "bf16", "out": "f32", "add": False},
        # odd lengths, a decoder that goes on behind a prefix, fp32, added to what is there
        {"name": "bias grad odd f32", "op": "bias grad", "batch": 1, "heads": 12, "q": 333, "k": 517, "offset": 184, "buckets": 32, "far": 128,
         "both": False, "dtype": "f32", "out": "f32", "add": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "ln", "ln bwd", "bias", "bias grad"])
    dtype, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    if op == "adamw":
        count = _log(rng, 1, 300)
        return {"op": op, "set": "drawn", "shapes": rng.randrange(1 << 30), "count": count, "most": _log(rng, 1000, min(20_000_000, 250_000_000 // count * 10)),
                "dtype": dtype, "bits": rng.choice([8, 32]), "copy": rng.random() < 0.5}
    if op in ("ln", "ln bwd"):
        cols = _log(rng, 16, 16384)
        cols = cols if rng.random() < 0.3 else max(16, cols // 64 * 64)       # mostly what models have, odd ones among them
        case = {"op": op, "rows": _log(rng, 1, min(131_072, (1 << 29) // cols)), "cols": cols, "dtype": dtype, "out": out if op == "ln" else dtype,
                "weight": rng.choice(["f32", dtype]), "affine": rng.choice(["both", "both", "weight", "none"] if op == "ln" else ["both", "both", "weight"])}
        return case if op == "ln" else {**case, "add": rng.random() < 0.3}
    heads, both = _log(rng, 1, 64), rng.random() < 0.5
    most = (1 << 27) // heads
    q = 1 if rng.random() < 0.15 else _log(rng, 1, min(8192, most))
    k = _log(rng, max(1, q // 4), min(8192, max(1, most // q)))
    buckets = rng.choice([8, 32, 32, 64])
    case = {"op": op, "heads": heads, "q": q, "k": k, "offset": rng.choice([0, max(0, k - q)]), "buckets": buckets,
            "far": _log(rng, buckets, 1024), "both": both, "dtype": dtype, "out": out}
    return case if op == "bias" else {**case, "batch": rng.randint(1, max(1, min(16, most // (q * k)))), "add": rng.random() < 0.3}


# ---- inputs -------------------------------------------------------------------------------------

def _gpt2_like(hidden, ffn, layers, vocab, pos):
    per = [3 * hidden * hidden, hidden * hidden, hidden * ffn, hidden * ffn, 3 * hidden, hidden, ffn, hidden] + [hidden] * 4
    return [vocab * hidden, pos * hidden] + per * layers


def _sizes(case):
    """Lengths of the tensors of an adamw case."""
    if case["set"] == "toy":
        return [512 * 256, 256]
    if case["set"] == "ragged":
        return [513 * 1030, 1001, 33 * 65, 1, 7, 300]
    if case["set"] == "gpt2_medium":
        return _gpt2_like(1024, 4096, 24, 50257, 1024)
    # "drawn": `count` tensors from 1 to `most` elements, spread over the logarithm
    u = torch.rand(case["count"], generator=torch.Generator().manual_seed(case["shapes"]), dtype=torch.float64)
    return [max(1, int(x)) for x in torch.exp(u * math.log(case["most"])).tolist()]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _exponent(x, bias):
    """The biased exponent of the power of two that a block's values are stored as multiples of."""
    most = x.view(-1, BLOCK).abs().amax(1)
    return ((most.view(torch.int32) >> 23) - bias).clamp_(0, 254)


def _power(e):
    return torch.exp2((e - 127).double()).float()


def _adamw_inputs(case, seed):
    """Flat buffers in which every tensor starts at a multiple of BLOCK, and (start, length) of each tensor."""
    gen, places, total = _generator(seed), [], 0
    for n in _sizes(case):
        places.append((total, n))
        total += -(-n // BLOCK) * BLOCK
    at = torch.tensor([p for p, _ in places], device="cuda")
    length = torch.tensor([n for _, n in places], device="cuda")
    block = torch.arange(total // BLOCK, device="cuda") * BLOCK
    owner = torch.searchsorted(at, block, right=True) - 1
    inside = (torch.arange(BLOCK, device="cuda")[None] < (at + length)[owner][:, None] - block[:, None]).view(-1)
    # one spread for a tensor: log-uniform in [1e-5, 1e-2]
    spread = torch.exp(torch.rand(len(places), generator=gen, device="cuda") * math.log(1e3)) * 1e-5
    spread = spread[owner][:, None].expand(-1, BLOCK).reshape(-1) * inside
    new = lambda: torch.empty(total, device="cuda").normal_(0.0, 1.0, generator=gen)  # noqa: E731
    s = {"places": places, "p": new().mul_(0.02).mul_(inside), "g": new().mul_(spread).to(DT[case["dtype"]])}
    m, v = new().mul_(spread).mul_(0.3), new().square_().mul_(0.3).add_(0.7).mul_(spread).mul_(spread)
    if case["bits"] == 32:
        return {**s, "m": m, "v": v}
    em, ev = _exponent(m, 7), _exponent(v, 14)
    s["m"] = (m.view(-1, BLOCK) / _power(em)[:, None]).to(torch.float8_e4m3fn).view(-1)
    s["v"] = (v.view(-1, BLOCK) / _power(ev)[:, None]).to(torch.float8_e5m2).view(-1)
    s["m_scale"], s["v_scale"] = (e.to(torch.uint8).view(torch.float8_e8m0fnu) for e in (em, ev))
    return s


def _ln_inputs(case, seed):
    """Activations whose rows have a mean of their own and a few of whose columns are large."""
    gen, rows, cols = _generator(seed), case["rows"], case["cols"]
    new = lambda *s, std=1.0: torch.empty(*s, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
    large = 1.0 + 20.0 * (torch.rand(cols, generator=gen, device="cuda") < 0.01)
    x = new(rows, cols).mul_(large).add_(new(rows, 1, std=0.5)).to(DT[case["dtype"]])
    w = new(cols, std=0.1).add_(1.0).to(DT[case["weight"]]) if case["affine"] != "none" else None
    b = new(cols, std=0.1).to(DT[case["weight"]]) if case["affine"] == "both" else None
    s = {"x": x, "w": w, "b": b}
    if case["op"] == "ln bwd":
        s["dy"] = new(rows, cols, std=1e-3).to(DT[case["dtype"]])
        s["dw"] = new(cols, std=1e-2).to(w.dtype)
        s["db"] = new(cols, std=1e-2).to(w.dtype) if b is not None else None
        mean = torch.empty(rows, device="cuda")
        rstd = torch.empty(rows, device="cuda")
        for a in range(0, rows, 8192):
            part = x[a:a + 8192].double()
            mean[a:a + 8192] = part.mean(1)
            rstd[a:a + 8192] = torch.rsqrt(part.var(1, unbiased=False) + LN_EPS)
        s["mean"], s["rstd"] = mean, rstd
    return s


def _bias_inputs(case, seed):
    gen = _generator(seed)
    if case["op"] == "bias":
        return {"table": torch.empty(case["buckets"], case["heads"], device="cuda").normal_(0.0, 1.0, generator=gen).to(DT[case["dtype"]])}
    # the gradient that a softmax hands to its scores: a row's values add up to nothing
    shape = (case["heads"], case["q"], case["k"])
    dout = torch.empty(case["batch"], *shape, dtype=DT[case["dtype"]], device="cuda")
    for n in range(case["batch"]):
        p = torch.softmax(torch.empty(shape, device="cuda").normal_(0.0, 2.0, generator=gen), -1)
        d = torch.empty(shape, device="cuda").normal_(0.0, 1e-2, generator=gen)
        dout[n] = p * (d - (p * d).sum(-1, keepdim=True))
    return {"dout": dout, "dtable": torch.empty(case["buckets"], case["heads"], device="cuda").normal_(0.0, 1e-2, generator=gen).to(DT[case["out"]])}


def prepare(case, seed):
    s = {"adamw": _adamw_inputs, "ln": _ln_inputs, "ln bwd": _ln_inputs, "bias": _bias_inputs, "bias grad": _bias_inputs}[case["op"]](case, seed)
    s["case"], s["t"] = case, STEPS_BEFORE
    if case["op"] == "adamw":
        s["copy"] = torch.zeros(s["p"].shape, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
        if own:
            from paper_2307_02047_b200 import binding
            part = lambda x: [x[a:a + n] for a, n in s["places"]] if x is not None else None  # noqa: E731
            blocks = lambda x: [x[a // BLOCK:-(-(a + n) // BLOCK)] for a, n in s["places"]] if x is not None else None  # noqa: E731
            s["opt"] = binding.AdamWOptimizer(
                part(s["p"]), part(s["g"]), state_bits=case["bits"], m=part(s["m"]), v=part(s["v"]), m_scale=blocks(s.get("m_scale")),
                v_scale=blocks(s.get("v_scale")), bf16_copy=part(s["copy"]), seed=SEED, step_count=STEPS_BEFORE)
    return s


# ---- one pass, in plain operations ------------------------------------------------------------

def _mix(x):
    """Scrambles the 32 bits of every value (int32, wrapping)."""
    x = x ^ ((x >> 16) & 0xFFFF)
    x = x * -0x4498517B
    x = x ^ ((x >> 15) & 0x1FFFF)
    x = x * -0x5AB00AC5
    return x ^ ((x >> 16) & 0xFFFF)


def _int32(x):
    return (x & 0xFFFFFFFF) - ((x & 0x80000000) << 1)


def _random_bits(total, t):
    """32 bits for every element: element i of a tensor's block takes mix(block's key + i * 0x9E3779B9)."""
    key = torch.zeros(1, dtype=torch.int32, device="cuda")
    for word in (SEED & 0xFFFFFFFF, SEED >> 32, t & 0xFFFFFFFF, t >> 32):
        key = _mix((key ^ _int32(word)) + 0x3C6EF373)
    golden = _int32(0x9E3779B9)
    blocks = _mix(key + torch.arange(total // BLOCK, dtype=torch.int32, device="cuda") * golden)
    return _mix(blocks[:, None] + (torch.arange(BLOCK, dtype=torch.int32, device="cuda") * golden)[None]).view(-1)


def _to_bits(x, e, low, drop, r):
    """Magnitudes as the bits of a small float: `drop` bits of fp32 dropped after a random number is added to them;
    2^low brings the small type's exponents to fp32's, subnormal ones included."""
    y = x.abs().view(-1, BLOCK) * _power(254 - e)[:, None] * 2.0 ** low
    return (y.view(-1).view(torch.int32) + r) >> drop


def _plain_adamw(s):
    c, t = s["case"], s["t"]
    f32 = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")  # noqa: E731
    b1, c1, b2, c2 = (f32(x) for x in (HP["beta1"], 1 - HP["beta1"], HP["beta2"], 1 - HP["beta2"]))
    p, g = s["p"], s["g"].float()
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * _power(s["m_scale"].view(torch.uint8).int())[:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * _power(s["v_scale"].view(torch.uint8).int())[:, None]).view(-1)
    m = b1 * m + c1 * g
    v = b2 * v + c2 * (g * g)
    step = HP["lr"] / (1 - HP["beta1"] ** t)
    p.sub_(HP["lr"] * HP["weight_decay"] * p + step * (m / (torch.sqrt(v) * (1 - HP["beta2"] ** t) ** -0.5 + HP["eps"])))
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return p, s["m"], s["v"], s["copy"]
    em, ev = _exponent(m, 7), _exponent(v, 14)
    r = _random_bits(p.numel(), t)
    mbits = _to_bits(m, em, -120, 20, (r & 0xFFFF) * 16 + 8)
    mbits = mbits | ((m.view(torch.int32) >> 24) & 0x80)
    vbits = _to_bits(v, ev, -112, 21, ((r >> 16) & 0xFFFF) * 32 + 16)
    vbits = torch.where(v > 0, vbits.clamp(min=1), vbits)
    s["m"].view(torch.uint8).copy_(mbits)
    s["v"].view(torch.uint8).copy_(vbits)
    s["m_scale"].view(torch.uint8).copy_(em)
    s["v_scale"].view(torch.uint8).copy_(ev)
    return p, s["m"], s["v"], s["m_scale"], s["v_scale"], s["copy"]


def _plain_ln(s):
    c, x = s["case"], s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + LN_EPS)
    y = x * rstd
    if s["w"] is not None:
        y = y * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    return y.to(DT[c["out"]]), mean[:, 0], rstd[:, 0]


def _plain_ln_bwd(s):
    add, rstd = s["case"]["add"], s["rstd"][:, None]
    h = (s["x"].float() - s["mean"][:, None]) * rstd
    dy = s["dy"].float()
    dw = (dy * h).sum(0)
    s["dw"].copy_(s["dw"].float() + dw if add else dw)
    if s["db"] is not None:
        db = dy.sum(0)
        s["db"].copy_(s["db"].float() + db if add else db)
    d = dy * s["w"].float()
    dx = rstd * (d - d.mean(1, keepdim=True) - h * (d * h).mean(1, keepdim=True))
    return dx.to(DT[s["case"]["out"]]), s["dw"], s["db"]


def _buckets(c):
    """The bucket of every (query, key), [q, k]; the logarithms in 64 bits, and what lies at a border belongs above it."""
    rel = torch.arange(c["k"], device="cuda")[None] - torch.arange(c["q"], device="cuda")[:, None] - c["offset"]
    n = c["buckets"] // 2 if c["both"] else c["buckets"]
    first = n * (rel > 0) if c["both"] else 0
    d = rel.abs() if c["both"] else (-rel).clamp(min=0)
    near = n // 2
    far = near + (torch.log(d.clamp(min=1).double() / near) / math.log(c["far"] / near) * (n - near) + 1e-10).floor().long()
    return first + torch.where(d < near, d, far.clamp(max=n - 1))


def _plain_bias(s):
    c = s["case"]
    return s["table"].float().t().contiguous()[:, _buckets(c)].to(DT[c["out"]])


def _plain_bias_grad(s):
    c = s["case"]
    hot = (_buckets(c).view(-1, 1) == torch.arange(c["buckets"], device="cuda")).float()
    d = s["dout"].float().sum(0).view(c["heads"], -1)
    total = (d @ hot).t()
    s["dtable"].copy_(s["dtable"].float() + total if c["add"] else total)
    return s["dtable"]


def run(state):
    c = state["case"]
    state["t"] += 1
    if own:
        from paper_2307_02047_b200 import binding
        if c["op"] == "adamw":
            state["opt"].step(**HP)
            return [state[x] for x in ("p", "m", "v", "m_scale", "v_scale", "copy") if x in state]
        if c["op"] == "ln":
            return binding.layer_norm_forward(state["x"], state["w"], state["b"], LN_EPS, out_dtype=DT[c["out"]])
        if c["op"] == "ln bwd":
            dx = binding.layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["w"], grad_weight=state["dw"],
                                             grad_bias=state["db"], accumulate=c["add"])
            return dx, state["dw"], state["db"]
        if c["op"] == "bias":
            return binding.position_bias_forward(state["table"], c["q"], c["k"], c["offset"], bidirectional=c["both"], max_distance=c["far"],
                                                 out_dtype=DT[c["out"]])
        return binding.position_bias_backward(state["dout"], state["dtable"], c["offset"], bidirectional=c["both"], max_distance=c["far"],
                                              accumulate=c["add"])
    return {"adamw": _plain_adamw, "ln": _plain_ln, "ln bwd": _plain_ln_bwd, "bias": _plain_bias, "bias grad": _plain_bias_grad}[c["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n, blocks = sum(_sizes(case)), sum(-(-k // BLOCK) for k in _sizes(case))
        state = 16 * n if case["bits"] == 32 else 4 * n + 4 * blocks          # read and written
        return {"bytes": n * (8 + SIZE[case["dtype"]] + (2 if case["copy"] else 0)) + state, "flops": 15 * n}
    if case["op"] == "ln":
        n, params = case["rows"] * case["cols"], {"both": 2, "weight": 1, "none": 0}[case["affine"]]
        return {"bytes": n * (SIZE[case["dtype"]] + SIZE[case["out"]]) + params * case["cols"] * SIZE[case["weight"]] + 8 * case["rows"], "flops": 8 * n}
    if case["op"] == "ln bwd":
        n, params = case["rows"] * case["cols"], 2 if case["affine"] == "both" else 1
        moved = 1 + params * (2 if case["add"] else 1)                        # the weight, and its gradients
        return {"bytes": n * (2 * SIZE[case["dtype"]] + SIZE[case["out"]]) + moved * case["cols"] * SIZE[case["weight"]] + 8 * case["rows"], "flops": 12 * n}
    n, table = case["heads"] * case["q"] * case["k"], case["buckets"] * case["heads"]
    if case["op"] == "bias":
        return {"bytes": n * SIZE[case["out"]] + table * SIZE[case["dtype"]], "flops": n}
    return {"bytes": case["batch"] * n * SIZE[case["dtype"]] + table * SIZE[case["out"]] * (2 if case["add"] else 1), "flops": case["batch"] * n}


# ---- in 64 bits ------------------------------------------------------------------------------------

def _exact_hash(x):
    """The same scrambling on values 0 .. 2^32 - 1."""
    for shift, factor in ((16, 0xBB67AE85), (15, 0xA54FF53B)):
        x = ((x ^ (x >> shift)) * factor) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _exact_codes(x, r, top, smallest, fraction):
    """Stored values and scales: multiples of the type's spacing at each value, the next one up with the probability of what is left over."""
    rows = x.view(-1, BLOCK)
    most = rows.abs().amax(1)
    scale = torch.where(most > 0, torch.exp2(torch.floor(torch.log2(most.clamp(min=1e-300))) - top), 2.0 ** -127).clamp(min=2.0 ** -127)
    z = (rows.abs() / scale[:, None]).view(-1)
    spacing = torch.exp2(torch.frexp(z)[1].double().sub(1).clamp(min=smallest) - fraction)
    z = torch.floor(z / spacing + (r.double() + 0.5) / 65536) * spacing
    return z * torch.sign(x), scale


def _exact_adamw(case, seed):
    s, t = _adamw_inputs(case, seed), STEPS_BEFORE + 1
    p, g, m, v = (s[k].double() for k in ("p", "g", "m", "v"))
    if case["bits"] == 8:
        m, v = ((x.view(-1, BLOCK) * s[k].double()[:, None]).view(-1) for x, k in ((m, "m_scale"), (v, "v_scale")))
    m = m + (1 - HP["beta1"]) * (g - m)
    v = v + (1 - HP["beta2"]) * (g.square() - v)
    mhat, vhat = m / (1 - HP["beta1"] ** t), v / (1 - HP["beta2"] ** t)
    p = p * (1 - HP["lr"] * HP["weight_decay"]) - HP["lr"] * mhat / (vhat.sqrt() + HP["eps"])
    copy = p if case["copy"] else None
    if case["bits"] == 32:
        return p, m, v, copy
    key = torch.zeros(1, dtype=torch.int64, device="cuda")
    for word in (SEED % 2 ** 32, SEED // 2 ** 32, t, 0):
        key = _exact_hash(((key ^ word) + 0x3C6EF373) % 2 ** 32)
    place = torch.arange(p.numel(), device="cuda")
    golden = 0x9E3779B9
    r = _exact_hash((_exact_hash((key + place // BLOCK * golden) % 2 ** 32) + place % BLOCK * golden) % 2 ** 32)
    mc, ms = _exact_codes(m, r % 65536, 7, -6, 3)
    vc, vs = _exact_codes(v, r // 65536, 14, -14, 2)
    return p, mc, torch.where((v > 0) & (vc == 0), 2.0 ** -16, vc), ms, vs, copy


def exact(case, seed):
    if case["op"] == "adamw":
        return _exact_adamw(case, seed)
    if case["op"] in ("ln", "ln bwd"):
        s = _ln_inputs(case, seed)
        step = max(1, (1 << 25) // case["cols"])
        if case["op"] == "ln":
            y = torch.empty(case["rows"], case["cols"], dtype=torch.float64, device="cuda")
            mean, rstd = torch.empty(case["rows"], dtype=torch.float64, device="cuda"), torch.empty(case["rows"], dtype=torch.float64, device="cuda")
            for a in range(0, case["rows"], step):
                x = s["x"][a:a + step].double()
                var, mu = torch.var_mean(x, 1, correction=0)
                mean[a:a + step], rstd[a:a + step] = mu, (var + LN_EPS) ** -0.5
                h = (x - mu[:, None]) / (var + LN_EPS).sqrt()[:, None]
                y[a:a + step] = h * (s["w"].double() if s["w"] is not None else 1.0) + (s["b"].double() if s["b"] is not None else 0.0)
            return y, mean, rstd
        w = s["w"].double()
        dx = torch.empty(case["rows"], case["cols"], dtype=torch.float64, device="cuda")
        dw = s["dw"].double() if case["add"] else torch.zeros_like(w)
        db = s["db"].double() if case["add"] and s["db"] is not None else torch.zeros_like(w)
        for a in range(0, case["rows"], step):
            rstd = s["rstd"][a:a + step, None].double()
            h = (s["x"][a:a + step].double() - s["mean"][a:a + step, None].double()) * rstd
            dy = s["dy"][a:a + step].double()
            dw += torch.einsum("rc,rc->c", dy, h)
            db += dy.sum(0)
            first, second = dy @ w, torch.einsum("rc,rc,c->r", dy, h, w)
            dx[a:a + step] = (dy * w - (first[:, None] + h * second[:, None]) / case["cols"]) * rstd
        return dx, dw, db if s["db"] is not None else None
    s, by_diagonal = _bias_inputs(case, seed), {}
    n = case["buckets"] // 2 if case["both"] else case["buckets"]
    near = n // 2

    def bucket(rel):
        d = abs(rel) if case["both"] else max(-rel, 0)
        if d >= near:          # the largest step up with near (far / near)^(step / (n - near)) <= d, in whole numbers
            k = 0
            while k < n - near - 1 and case["far"] ** (k + 1) * near ** (n - near - k - 1) <= d ** (n - near):
                k += 1
            d = near + k
        return d + (n if case["both"] and rel > 0 else 0)

    for rel in range(1 - case["q"], case["k"]):
        by_diagonal[rel] = bucket(rel - case["offset"])
    if case["op"] == "bias":
        line = s["table"].double()[torch.tensor([by_diagonal[rel] for rel in range(1 - case["q"], case["k"])], device="cuda")].t().contiguous()
        place = torch.arange(case["k"], device="cuda")[None] - torch.arange(case["q"], device="cuda")[:, None] + case["q"] - 1
        return line[:, place]
    d, total = s["dout"], s["dtable"].double().clone() if case["add"] else torch.zeros(case["buckets"], case["heads"], dtype=torch.float64, device="cuda")
    d = d.double().sum(0)
    for rel, b in by_diagonal.items():
        total[b] += d.diagonal(rel, 1, 2).sum(-1)
    return total
