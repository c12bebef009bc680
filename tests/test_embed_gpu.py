"""Embedding lookup and its gradient against the formulas in 64 bits.

Tolerances, from the arithmetic.  Forward: one product, one rounding: equal bit for bit to the
fp32 product rounded to the output's type.  Backward: n fp32 additions in some order, the product
with the scale and the old value round by 2^-24 each, so before the store the value lies within
  e = (n + 3) 2^-24 (|scale| sum |dY| + |old|)
of the exact one, and what is stored lies between ref - e and ref + e, both rounded to the output's
type (rounding keeps the order)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
SENT = 1232.0


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2307_02047_b200 import binding
    assert torch.cuda.is_available()
    return torch, binding


def _dt(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}[name]


def _strided(torch, rows, cols, dtype, gap, offset):
    """A rows x cols view with row stride cols + gap, `offset` elements into a guarded buffer."""
    ld = cols + gap
    arena = torch.full((64 + offset + max(rows, 1) * ld + 64,), SENT, dtype=dtype, device="cuda")
    return arena, arena[64 + offset:64 + offset + max(rows, 1) * ld].view(-1, ld)[:rows, :cols]


def _outside_untouched(torch, arena, view):
    mask = torch.ones_like(arena, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset() - arena.storage_offset()).fill_(False)
    return bool((arena[mask] == SENT).all())


def _ids(torch, kind, tokens, rows, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "same":
        ids = torch.full((tokens,), rows - 1, device="cuda", dtype=torch.int64)
    elif kind == "none":
        ids = torch.full((tokens,), -1, device="cuda", dtype=torch.int64)
        ids[::2] = rows
    elif kind == "hot":                      # a few rows have nearly all tokens, some tokens are padding
        u = torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * np.log(rows + 1)) - 1).long().clamp_(0, rows - 1)
        ids[torch.rand(tokens, generator=g, device="cuda") < 0.1] = -100
    else:
        ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    if dtype == torch.int64 and tokens > 3 and kind != "same":
        ids[tokens // 2], ids[1] = 2 ** 40, -(2 ** 62)
    return ids.to(dtype)


def _reference(dy, ids, old, rows, scale, padding, accumulate):
    """dW in float64, and the elementwise bound on sum |.| that the tolerance uses."""
    ids = ids.reshape(-1).cpu().numpy().astype(np.int64)
    dy = dy.reshape(-1, dy.shape[-1]).double().cpu().numpy()
    ok = (ids >= 0) & (ids < rows)
    if padding is not None:
        ok &= ids != padding
    ref, mag = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1]))
    np.add.at(ref, ids[ok], dy[ok])
    np.add.at(mag, ids[ok], np.abs(dy[ok]))
    count = np.bincount(ids[ok], minlength=rows)
    ref, mag = scale * ref, abs(scale) * mag
    if accumulate:
        old = old.double().cpu().numpy()
        ref, mag = ref + old, mag + np.abs(old)
    return ref, mag, count


def _check_grad(got, ref, mag, count):
    import torch
    e = (count[:, None] + 3) * 2.0 ** -24 * mag
    low, high = (torch.from_numpy(x).to(got.dtype).double().numpy() for x in (ref - e, ref + e))
    got = got.double().cpu().numpy()
    assert np.all((low <= got) & (got <= high)), f"{np.sum((got < low) | (got > high))} of {got.size} out of bounds"


CASES = [   # tokens, rows, cols, ids, kind, gap, offset
    (0, 5, 8, "i64", "any", 0, 0), (1, 1, 1, "i32", "any", 0, 0), (2, 3, 2, "i64", "same", 0, 1),
    (33, 512, 256, "i64", "any", 0, 0), (31, 7, 257, "i32", "hot", 0, 0), (64, 511, 255, "i64", "any", 1, 0),
    (1000, 513, 1030, "i32", "hot", 0, 0), (1025, 100, 772, "i64", "hot", 4, 4), (1024, 2, 64, "i32", "any", 0, 8),
    (4096, 1000, 128, "i64", "any", 0, 0), (4097, 30522, 96, "i64", "hot", 0, 0), (5000, 300, 40, "i32", "same", 8, 0),
    (3000, 300, 520, "i32", "none", 0, 0), (20000, 50257, 24, "i64", "hot", 0, 0), (70001, 262200, 8, "i32", "hot", 0, 0),
    (9000, 50, 7, "i64", "hot", 0, 3), (40000, 3, 256, "i32", "any", 0, 0), (2048, 600, 2048, "i64", "hot", 16, 16),
]


@pytest.mark.parametrize("tdt,odt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("k", range(len(CASES)))
def test_forward_is_the_rounded_product(env, tdt, odt, k):
    torch, binding = env
    tokens, rows, cols, idt, kind, gap, offset = CASES[k]
    _, table = _strided(torch, rows, cols, _dt(torch, tdt), gap, offset)
    table.normal_(0, 0.02)
    ids = _ids(torch, kind, tokens, rows, _dt(torch, idt), k)
    arena, out = _strided(torch, tokens, cols, _dt(torch, odt), gap, offset)
    for scale in (1.0, 22.627):
        binding.embed_forward(table, ids, scale, out=out)
        ok = (ids >= 0) & (ids < rows)
        want = table[torch.where(ok, ids, 0).long()].float() * torch.tensor(scale, dtype=torch.float32)
        want = torch.where(ok[:, None], want, 0.0).to(out.dtype)
        assert torch.equal(out, want)
        assert _outside_untouched(torch, arena, out)


@pytest.mark.parametrize("ydt,gdt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("k", range(len(CASES)))
def test_gradient_against_64_bits(env, ydt, gdt, k):
    torch, binding = env
    tokens, rows, cols, idt, kind, gap, offset = CASES[k]
    torch.manual_seed(k)
    _, dy = _strided(torch, tokens, cols, _dt(torch, ydt), gap, offset)
    dy.normal_(0, 1e-3)
    ids = _ids(torch, kind, tokens, rows, _dt(torch, idt), k)
    for scale, padding, accumulate in ((1.0, None, False), (-3.5, 0, False), (22.627, rows - 1, True), (0.5, None, True)):
        arena, grad = _strided(torch, rows, cols, _dt(torch, gdt), gap, offset)
        grad.normal_(0, 1e-2)
        old = grad.clone()
        got = binding.embed_backward(dy, ids, grad, scale, padding_row=padding, accumulate=accumulate)
        assert got is grad
        ref, mag, count = _reference(dy, ids, old, rows, scale, padding, accumulate)
        _check_grad(grad, ref, mag, count)
        assert _outside_untouched(torch, arena, grad)
        untouched = torch.from_numpy(count == 0).cuda()
        assert torch.equal(grad[untouched], old[untouched] if accumulate else torch.zeros_like(old[untouched]))


@pytest.mark.parametrize("tokens,rows,kind", [
    (1, 1000, "any"), (511, 1000, "hot"), (512, 1000, "any"), (513, 1000, "hot"), (300, (1 << 22) + 5, "any"), (4096, 5, "hot"),
    (4097, 70000, "any"), (151_553, 1000, "hot"), (620_001, 300, "hot"), (620_001, 300_000, "any"), (100_000, 1, "any"), (200_000, 40, "same"),
])
def test_sorting_of_every_length(env, tokens, rows, kind):
    """Every way the tokens are sorted: whole numbers small enough that fp32 sums are exact, so the
    result must equal the exact one; few columns, many tokens."""
    torch, binding = env
    ids = _ids(torch, kind, tokens, rows, torch.int32, tokens)
    dy = torch.randint(-3, 4, (tokens, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
    got = binding.embed_backward(dy, ids, torch.empty(rows, 2, device="cuda"))
    ok = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, 2, device="cuda", dtype=torch.int64)
    want.index_add_(0, ids[ok].long(), dy[ok].long())
    assert torch.equal(got, want.float())


def test_gradient_against_differences(env):
    """The lookup is linear in the table: <dW, E> = <c, out(W + E) - out(W - E)> / 2 for any E.
    The right side rounds each product by 2^-24 of an output; the left each sum as above."""
    torch, binding = env
    torch.manual_seed(5)
    rows, cols, tokens, scale = 301, 136, 2000, 4.0
    ids = _ids(torch, "hot", tokens, rows, torch.int64, 5)
    W, c = torch.randn(rows, cols, device="cuda"), torch.randn(tokens, cols, device="cuda")
    dW = binding.embed_backward(c, ids, torch.empty_like(W), scale)
    for seed in range(4):
        E = torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        up, down = W + E, W - E
        step = (up.double() - down.double()) / 2                    # what E became in fp32
        diff = (binding.embed_forward(up, ids, scale).double() - binding.embed_forward(down, ids, scale).double()) / 2
        right, left = (c.double() * diff).sum(), (dW.double() * step).sum()
        size = float((c.double().abs() * scale * (W.abs().max() + E.abs()).max()).sum())
        assert abs(float(left - right)) <= size * (tokens + 4) * 2.0 ** -24


def test_non_finite_values_stay_in_their_rows(env):
    torch, binding = env
    rows, cols = 40, 24
    ids = torch.arange(100, device="cuda") % 20
    ids[7] = -1
    dy = torch.ones(100, cols, device="cuda")
    dy[3, 5], dy[4, 6], dy[7] = float("inf"), float("nan"), float("nan")      # token 7 is padding
    for dt in (torch.float32, torch.bfloat16):
        g = binding.embed_backward(dy.to(dt), ids, torch.full((rows, cols), float("nan"), device="cuda", dtype=dt))
        bad = ~g.isfinite()
        assert bad.nonzero().tolist() == [[3, 5], [4, 6]] and bool(g[3, 5].isinf()) and bool((g[20:] == 0).all())
    table = torch.full((rows, cols), float("nan"), device="cuda")
    table[2] = 1.0
    out = binding.embed_forward(table, torch.tensor([2, -1, 3, rows], device="cuda"))
    assert bool((out[0] == 1).all()) and bool((out[1] == 0).all()) and bool(out[2].isnan().all()) and bool((out[3] == 0).all())


def test_shapes_streams_and_reproducibility(env):
    torch, binding = env
    torch.manual_seed(9)
    rows, cols = 5000, 320
    ids = _ids(torch, "hot", 6 * 700, rows, torch.int64, 3).view(6, 700)
    table = torch.randn(rows, cols, device="cuda")
    out = binding.embed_forward(table, ids, 2.0, out_dtype=torch.bfloat16)
    assert out.shape == (6, 700, cols) and out.dtype == torch.bfloat16
    one = binding.embed_forward(table, ids[0, 5].clone())
    assert one.shape == (cols,)
    dy = torch.randn(6, 700, cols, device="cuda")
    first = binding.embed_backward(dy, ids, torch.empty(rows, cols, device="cuda")).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    grads = []
    for k in range(8):                      # two streams, workspaces of their own
        with torch.cuda.stream(side if k % 2 else torch.cuda.default_stream()):
            grads.append(binding.embed_backward(dy, ids, torch.empty(rows, cols, device="cuda")))
    torch.cuda.synchronize()
    assert all(torch.equal(g, first) for g in grads)
    graph = torch.cuda.CUDAGraph()
    g = torch.empty(rows, cols, device="cuda")
    with torch.cuda.graph(graph):
        binding.embed_backward(dy, ids, g)
    g.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g, first)


def test_large_offsets(env):
    """Row offsets beyond 2^31 elements in the table, and token offsets in the data."""
    torch, binding = env
    rows, cols = 70_000, 40_000                                   # 2.8e9 elements, 5.6 GB
    table = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    table[rows - 1], table[rows - 3] = 3.0, 5.0
    ids = torch.tensor([rows - 1, 0, rows - 3, rows], device="cuda")
    out = binding.embed_forward(table, ids, 0.5)
    assert out.float().mean(1).tolist() == [1.5, 0.0, 2.5, 0.0]
    table.fill_(9.0)
    binding.embed_backward(out, ids, table, 2.0)
    assert bool((table[rows - 1] == 3).all()) and bool((table[rows - 3] == 5).all())
    table[rows - 1], table[rows - 3] = 0.0, 0.0
    assert int(table.count_nonzero()) == 0
    del out
    dy = table                                                     # 70000 tokens of 40000 columns, read far out
    dy[-1] = 1.0
    dy[-2] = 0.25
    ids = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    ids[-1], ids[-2] = 2, 2
    g = binding.embed_backward(dy, ids, torch.empty(3, cols, device="cuda"))
    assert g.mean(1).tolist() == [0.0, 0.0, 1.25]


def test_refusals(env):
    torch, binding = env
    t, ids = torch.ones(10, 8, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.int64)
    y = torch.ones(4, 8, device="cuda")

    def refused(status, call):
        with pytest.raises(binding.CameError) as e:
            call()
        assert e.value.status == status

    refused(binding.CAME_ERR_DTYPE, lambda: binding.embed_forward(t.double(), ids))
    refused(binding.CAME_ERR_DTYPE, lambda: binding.embed_forward(t, ids.float()))
    refused(binding.CAME_ERR_DTYPE, lambda: binding.embed_forward(t, ids, out=torch.empty_like(y), out_dtype=torch.bfloat16))
    refused(binding.CAME_ERR_DEVICE, lambda: binding.embed_forward(t.cpu(), ids))
    refused(binding.CAME_ERR_DEVICE, lambda: binding.embed_forward(t, ids.cpu()))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_forward(t[0], ids))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_forward(t, ids, out=y[:3]))
    refused(binding.CAME_ERR_UNSUPPORTED, lambda: binding.embed_forward(t.t(), ids))
    refused(binding.CAME_ERR_UNSUPPORTED, lambda: binding.embed_forward(t, torch.zeros(8, device="cuda", dtype=torch.int64)[::2]))
    refused(binding.CAME_ERR_HPARAM, lambda: binding.embed_forward(t, ids, float("inf")))
    refused(binding.CAME_ERR_OVERLAP, lambda: binding.embed_forward(t, ids, out=t[2:6]))
    refused(binding.CAME_ERR_OVERLAP, lambda: binding.embed_backward(t[2:6], ids, t))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(y, ids, t, padding_row=10))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(y, ids, t, padding_row=-1))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(y[:3], ids, t))
    refused(binding.CAME_ERR_SHAPE, lambda: binding.embed_backward(torch.ones(8, device="cuda").expand(4, 8), ids, t))
    e = binding.came_embed(t.data_ptr(), y.data_ptr(), ids.data_ptr(), 10, 8, 4, 8, 8, 0, 1.0, 0, 0, 1, 0, 0)
    ws = torch.empty(binding.came_embed_workspace(e), dtype=torch.uint8, device="cuda")
    refused(binding.CAME_ERR_SHAPE, lambda: binding.came_embed_backward(e, ws.data_ptr(), ws.numel() - 1))
    refused(binding.CAME_ERR_NULL, lambda: binding.came_embed_backward(e, None, ws.numel()))
    assert bool((t == 1).all())
