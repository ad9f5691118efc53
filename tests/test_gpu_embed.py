"""Embedding lookup and its gradient against their formulas in 64 bits, on the GPU.

A result is scale * a table's element, or scale * a sum (+ base), rounded once: off by half a step of its type (2^-8 for
bf16, 2^-24 for fp32), plus for a sum of n terms at most n additions in fp32, the product and the last addition:
(n + 3) * 2^-24 * scale * sum |terms| + 2^-24 |base|."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
HALF_STEP = {F32: U32, BF16: U16}


@pytest.fixture(scope="module")
def kt():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import binding
    torch.cuda.set_device(0)
    return binding


def placed(x, layout):
    """Contiguous; with a longer stride (aligned rows); or at an odd address and stride, NaN between the rows."""
    if layout == "plain":
        return x.cuda()
    pad, shift = (16, 0) if layout == "strided" else (3, 1)
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def untouched_around(view):
    if view.is_contiguous():
        return True
    flat = torch.empty(0, dtype=view.dtype, device="cuda").set_(view.untyped_storage())
    mask = torch.ones_like(flat, dtype=torch.bool)
    idx = view.storage_offset() + torch.arange(view.size(0), device="cuda")[:, None] * view.stride(0) + torch.arange(view.size(1), device="cuda")
    mask[idx.flatten()] = False
    return bool(torch.isnan(flat[mask].float()).all())


def text(gen, tokens, vocab, kind):
    if kind == "one":                                  # a text of one token
        return torch.full((tokens,), vocab // 2)
    ids = torch.randint(vocab, (tokens,), generator=gen)
    if kind == "skewed":
        ids = (torch.exp(torch.rand(tokens, generator=gen, dtype=torch.float64) * torch.log(torch.tensor(float(vocab)))) - 1).long().clamp(0, vocab - 1)
    if kind == "unknown":                              # padding, and ids past the table
        ids[::3], ids[1::5], ids[-1] = -1, vocab, 2 ** 40
    return ids


SHAPES = [(1, 1, 1), (1, 7, 5), (3, 16, 1), (64, 128, 1000), (77, 500, 8000), (999, 130, 300), (2000, 1032, 149), (33, 2050, 50257), (5, 4096, 7)]


@pytest.mark.parametrize("tokens,cols,vocab", SHAPES)
@pytest.mark.parametrize("wtype,otype,layout", [(F32, F32, "plain"), (BF16, BF16, "strided"), (F32, BF16, "odd"), (BF16, F32, "plain")])
def test_forward(kt, tokens, cols, vocab, wtype, otype, layout):
    gen = torch.Generator().manual_seed(tokens + cols)
    weight = placed(torch.randn(vocab, cols, generator=gen).to(wtype), layout)
    ids = text(gen, tokens, vocab, "unknown" if tokens > 1 else "plain").cuda()
    out = placed(torch.full((tokens, cols), 7.0, dtype=otype), layout)
    kt.kt_embed_forward(ids, weight, out, scale=1.7)
    known, pad = (ids >= 0) & (ids < vocab), ids < 0
    want = torch.tensor(1.7, dtype=F32).double().cuda() * weight.double()[ids.clamp(0, vocab - 1)]
    assert (out[pad] == 0).all() and torch.isnan(out[~known & ~pad]).all()
    assert ((out.double() - want).abs() <= (HALF_STEP[otype] + 2 * U32) * want.abs())[known].all()
    assert untouched_around(out)


def gradient(dout, ids, vocab, scale, base):
    known = (ids >= 0) & (ids < vocab)
    at, rows = ids[known], dout.double()[known]
    sums, sizes = (torch.zeros(vocab, dout.size(1), dtype=torch.float64, device="cuda") for _ in range(2))
    sums.index_add_(0, at, rows)
    sizes.index_add_(0, at, rows.abs())
    count = torch.bincount(at, minlength=vocab)[:, None]
    scale = torch.tensor(scale, dtype=F32).double().cuda()
    want = scale * sums + (base.double() if base is not None else 0.0)
    slack = (count + 3) * U32 * scale * sizes + (U32 * base.double().abs() if base is not None else 0.0)
    return want, slack


@pytest.mark.parametrize("tokens,cols,vocab,kind", [(1, 1, 1, "plain"), (1, 9, 5, "plain"), (31, 16, 3, "plain"), (33, 500, 40, "unknown"), (64, 128, 1000, "one"), (999, 130, 300, "skewed"),
                                                    (5000, 72, 149, "one"), (4097, 1032, 149, "unknown"), (3000, 2056, 8001, "skewed"), (20000, 64, 50257, "skewed"), (3000, 24, 310000, "skewed"),
                                                    (40000, 16, 7, "plain"), (300, 16, 30000, "skewed"), (2048, 511, 90000, "skewed"), (200, 4096, 5, "unknown"), (2049, 8, 20, "one")])
@pytest.mark.parametrize("dtype,wtype,layout,base", [(F32, F32, "plain", None), (BF16, BF16, "strided", "other"), (BF16, F32, "odd", "itself"), (F32, BF16, "plain", "itself")])
def test_gradient(kt, tokens, cols, vocab, kind, dtype, wtype, layout, base):
    gen = torch.Generator().manual_seed(tokens * 3 + cols)
    dout = placed(torch.randn(tokens, cols, generator=gen).to(dtype), layout)
    ids = text(gen, tokens, vocab, kind).cuda()
    dw = placed(torch.randn(vocab, cols, generator=gen).to(wtype), layout)
    before = {None: None, "other": placed(dw.cpu(), layout), "itself": dw}[base]
    kept = None if before is None else before.clone()
    want, slack = gradient(dout, ids, vocab, 0.3, kept)
    work = torch.full((kt.kt_embed_workspace(tokens, cols, vocab),), 255, dtype=torch.uint8, device="cuda")
    kt.kt_embed_backward(dout, ids, dw, work, scale=0.3, base=before)
    assert ((dw.double() - want).abs() <= HALF_STEP[wtype] * (want.abs() + slack) + slack).all()
    assert untouched_around(dw)
    seen = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    seen[ids[(ids >= 0) & (ids < vocab)]] = True
    rest = dw[~seen]
    assert torch.equal(rest, torch.zeros_like(rest) if kept is None else kept[~seen])
    if base != "itself":
        again = torch.empty_like(dw)
        kt.kt_embed_backward(dout, ids, again, work, scale=0.3, base=before)
        assert torch.equal(again, dw)


def test_no_tokens(kt):
    dw, base = torch.full((9, 24), 3.0, device="cuda"), torch.randn(9, 24, device="cuda")
    ids, dout = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, 24, device="cuda")
    work = torch.empty(kt.kt_embed_workspace(0, 24, 9), dtype=torch.uint8, device="cuda")
    kt.kt_embed_backward(dout, ids, dw, work, base=base)
    assert torch.equal(dw, base)
    kt.kt_embed_backward(dout, ids, dw, work)
    assert (dw == 0).all()
    kt.kt_embed_forward(ids, base, dout)


def test_gradient_is_that_of_the_lookup(kt):
    """The lookup is linear in the table, so a difference is exact but for rounding: <dout, lookup(w + d) - lookup(w)> = <dw, d>."""
    gen = torch.Generator().manual_seed(5)
    ids = text(gen, 700, 90, "skewed").cuda()
    w, d, dout = (torch.randn(n, 40, generator=gen).cuda() for n in (90, 90, 700))
    out = [torch.empty(700, 40, device="cuda") for _ in range(2)]
    kt.kt_embed_forward(ids, w, out[0], scale=2.0)
    kt.kt_embed_forward(ids, w + d, out[1], scale=2.0)
    dw = torch.empty_like(w)
    kt.kt_embed_backward(dout, ids, dw, torch.empty(kt.kt_embed_workspace(700, 40, 90), dtype=torch.uint8, device="cuda"), scale=2.0)
    left, right = (dout.double() * (out[1].double() - out[0].double())).sum(), (dw.double() * d.double()).sum()
    # rounding: w + d and both products by 2^-24 of some 10 (values), dw by 700 * 2^-24 of its terms
    sizes = (dout.abs().double() * 12).sum()
    assert (left - right).abs() <= 800 * U32 * sizes


def test_captured_beside_other_streams(kt):
    """A recorded call reads what its inputs hold when it is replayed, on whatever stream."""
    gen = torch.Generator().manual_seed(8)
    ids, dout, dw = text(gen, 500, 300, "skewed").cuda(), torch.randn(500, 256, generator=gen).cuda(), torch.empty(300, 256, device="cuda")
    work = torch.empty(kt.kt_embed_workspace(500, 256, 300), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kt.kt_embed_backward(dout, ids, dw, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kt.kt_embed_backward(dout, ids, dw, work)
    for _ in range(3):
        ids.copy_(text(gen, 500, 300, "skewed"))
        dout.copy_(torch.randn(500, 256, generator=gen))
        graph.replay()
        want, slack = gradient(dout, ids, 300, 1.0, None)
        assert ((dw.double() - want).abs() <= U32 * (want.abs() + slack) + slack).all()


def test_a_table_of_the_largest_size(kt):
    """Offsets past 2^31 elements, and more CTAs than SMs for the list."""
    tokens, cols, vocab = 600, 144, 2 ** 24
    gen = torch.Generator().manual_seed(11)
    ids = torch.randint(vocab - 1000, vocab, (tokens,), generator=gen).cuda()
    ids[:7] = torch.tensor([0, 1, vocab - 1, vocab - 1, -1, vocab, 5])
    dout = torch.randn(tokens, cols, generator=gen).to(BF16).cuda()
    dw = torch.full((vocab, cols), 3.0, dtype=BF16, device="cuda")
    work = torch.empty(kt.kt_embed_workspace(tokens, cols, vocab), dtype=torch.uint8, device="cuda")
    kt.kt_embed_backward(dout, ids, dw, work)
    known = (ids >= 0) & (ids < vocab)
    rows, at = torch.unique(ids[known], return_inverse=True)
    want = torch.zeros(len(rows), cols, dtype=torch.float64, device="cuda").index_add_(0, at, dout[known].double())
    assert ((dw[rows].double() - want).abs() <= U16 * want.abs() + 16 * U32 * dout.double().abs().max()).all()
    dw[rows] = 0
    assert not dw.any()
    dw[rows] = 1
    out = torch.empty(tokens, cols, dtype=BF16, device="cuda")
    kt.kt_embed_forward(ids, dw, out)
    assert (out[known] == 1).all()
