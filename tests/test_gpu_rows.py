"""Layer norm, activations and 8-bit checkpoints against their formulas in 64 bits, on the GPU.

Tolerances are derived, not fitted.  u32 = 2^-24 and u16 = 2^-8 (half a unit of bf16, doubled) are
the relative errors of one rounding.  A sum over a row is formed by at most `depth` additions one
after the other (16 in a thread, 5 across a warp, 16 across warps; wide rows cols / 512 + 21), so it
is off by at most depth * u32 * sum |terms|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (1, 7), (3, 16), (5, 127), (4, 128), (7, 130), (33, 512), (9, 520), (130, 1000), (17, 2048), (3, 4096),
          (2, 8192), (2, 8200), (3, 9001), (700, 72)]


@pytest.fixture(scope="module")
def kt():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import binding
    torch.cuda.set_device(0)
    return binding


def matrix(gen, rows, cols, dtype, layout="plain", std=1.5, mean=0.3):
    """A rows x cols matrix: contiguous, with a longer stride (aligned rows), or at an odd address and stride."""
    x = (torch.randn(rows, cols, generator=gen) * std + mean).to(dtype)
    return placed(x, layout)


def placed(x, layout):
    rows, cols = x.shape
    if layout == "plain":
        return x.cuda()
    pad, shift = (16, 0) if layout == "strided" else (3, 1)
    buf = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def surroundings_untouched(view):
    """The padding of a strided result still holds the NaNs it was made with."""
    if view.is_contiguous():
        return True
    base = view.untyped_storage()
    flat = torch.empty(0, dtype=view.dtype, device="cuda").set_(base)
    mask = torch.ones_like(flat, dtype=torch.bool)
    idx = view.storage_offset() + torch.arange(view.size(0), device="cuda")[:, None] * view.stride(0) + torch.arange(view.size(1), device="cuda")
    mask[idx.flatten()] = False
    return bool(torch.isnan(flat[mask].float()).all())


def blank(like):
    out = placed(torch.full(like.shape, float("nan"), dtype=like.dtype), "plain")
    return out if like.is_contiguous() else placed(out.cpu(), "odd" if like.storage_offset() % 8 else "strided")


def depth(cols):
    return 40 if cols <= 8192 else cols / 512 + 40


def rounding(dtype):
    return U32 if dtype == F32 else U16


def checkpoint(kt, rows, cols):
    return (torch.full((rows, kt.kt_ckpt_pitch(cols)), 77, dtype=torch.int8, device="cuda"),
            torch.full((rows, kt.kt_ckpt_blocks(cols)), -1.0, device="cuda"))


def decode(codes, scales, cols):
    at = torch.arange(cols, device=codes.device) // 128
    return codes[:, :cols].double() * scales.double()[:, at]


def encode_exactly(x):
    """Codes and scales of fp32 values, in the operations that the header names."""
    rows, cols = x.shape
    n = -(-cols // 128)
    b = torch.nn.functional.pad(x, (0, n * 128 - cols)).view(rows, n, 128)
    top = b.abs().amax(2)
    used = top >= 2.0 ** -100
    codes = torch.round(b * torch.where(used, 127.0 * (1.0 / top), 0.0)[..., None])
    return codes.view(rows, -1)[:, :cols], torch.where(used, top * torch.tensor(1.0 / 127.0, dtype=F32, device=x.device), 0.0)


@pytest.mark.parametrize("layout", ["plain", "strided", "odd"])
@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(kt, rows, cols, dtype, pdtype, layout):
    gen = torch.Generator().manual_seed(rows * 10007 + cols)
    x, dout = matrix(gen, rows, cols, dtype, layout), matrix(gen, rows, cols, dtype, layout)
    w, b = (torch.randn(cols, generator=gen).to(pdtype).cuda() for _ in range(2))
    out, mean, rstd = blank(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    codes, scales = checkpoint(kt, rows, cols)
    eps = 1e-5
    kt.kt_norm_forward(x, w, b, out, mean, rstd, eps, codes, scales)

    X, W, B, D = x.double(), w.double(), b.double(), dout.double()
    m = X.mean(1, keepdim=True)
    var = (X - m).square().mean(1, keepdim=True)
    r = (var + eps).rsqrt()
    u = (X - m) * r
    # mean: a sum's error over cols; the difference x - mean is rounded once; rstd: a relative error of a
    # sum of squares (half of it), of the shifted mean (second order) and of two more roundings
    e_mean = depth(cols) * U32 * X.abs().mean(1, keepdim=True)
    e_rstd = r * (U32 * (depth(cols) + 8) + e_mean * r)
    assert ((mean[:, None].double() - m).abs() <= e_mean + U32 * m.abs()).all()
    assert ((rstd[:, None].double() - r).abs() <= e_rstd).all()
    e_u = (e_mean + U32 * (X - m).abs()) * r + (X - m).abs() * e_rstd + U32 * u.abs()
    y = u * W + B
    assert ((out.double() - y).abs() <= e_u * W.abs() + 2 * U32 * (u * W).abs() + rounding(dtype) * y.abs() + U32 * B.abs()).all()
    assert surroundings_untouched(out)
    # the checkpoint: within half a step of u, padding columns zero
    step = scales.double()[:, torch.arange(cols, device="cuda") // 128]
    assert ((decode(codes, scales, cols) - u).abs() <= step * (0.5 + 127 * 4 * U32) + e_u).all()
    assert not codes[:, cols:].any()

    for kept in (False, True):
        dx, dw, db = blank(x), torch.full((cols,), math.nan, dtype=pdtype, device="cuda"), torch.full((cols,), math.nan, dtype=pdtype, device="cuda")
        work = torch.full((max(1, kt.kt_norm_workspace(rows, cols)),), 255, dtype=torch.uint8, device="cuda")
        src = {"codes": codes, "scales": scales} if kept else {"x": x, "mean": mean}
        kt.kt_norm_backward(dout, w, rstd, dx, dw, db, work, **src)
        M, R = mean[:, None].double(), rstd[:, None].double()
        un = decode(codes, scales, cols) if kept else (X - M) * R
        g = D * W
        s1, s2 = g.mean(1, keepdim=True), (g * un).mean(1, keepdim=True)
        want = (g - s1 - un * s2) * R
        d = depth(cols) + 8
        e = R * d * U32 * (g.abs() + g.abs().mean(1, keepdim=True) + un.abs() * (g * un).abs().mean(1, keepdim=True))
        assert ((dx.double() - want).abs() <= e + rounding(dtype) * want.abs()).all()
        assert surroundings_untouched(dx)
        n = rows + 24                                  # additions of a column's sum, at the very most
        for got, terms in ((dw, D * un), (db, D)):
            assert ((got.double() - terms.sum(0)).abs() <= (n + 4) * U32 * terms.abs().sum(0) + rounding(pdtype) * terms.sum(0).abs()).all()


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1000, 1029, 1500, 2000, 2500, 2561, 2700, 4000, 5120, 5121, 6000, 8000])
def test_norm_on_each_number_of_threads(kt, cols, dtype, layout):
    """Rows of 64, 96, 128, 160, 192, 256, 320, 384 and 512 threads; one cluster, and a row of partial sums to a CTA."""
    for rows in (21, 330):
        test_norm(kt, rows, cols, dtype, F32, layout)


def test_norm_against_differences(kt):
    """dx, dweight and dbias against central differences of the forward kernel itself (fp32).

    L = sum(y * dout) is summed in 64 bits.  With step h a difference is off by h^2 / 6 times the third
    derivative (the rows have unit spread: below 20 here) and by the rounding of 2 * 24 outputs,
    each below 8 * U32 * |y dout|, over 2 h."""
    gen = torch.Generator().manual_seed(3)
    rows, cols, h = 3, 24, 2.0 ** -7
    x, dout = matrix(gen, rows, cols, F32), matrix(gen, rows, cols, F32)
    w, b = (torch.randn(cols, generator=gen).cuda() for _ in range(2))
    out, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def loss(x_, w_, b_):
        kt.kt_norm_forward(x_, w_, b_, out, mean, rstd)
        return float((out.double() * dout.double()).sum())

    loss(x, w, b)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    work = torch.empty(kt.kt_norm_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    kt.kt_norm_backward(dout, w, rstd, dx, dw, db, work, x=x, mean=mean)
    tol = h * h / 6 * 20 + 2 * 24 * rows * 8 * U32 * 10 / (2 * h)
    for base, grad in ((x, dx), (w, dw), (b, db)):
        for i in range(0, base.numel(), 5):
            up, down = base.clone(), base.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            args = [tuple(t if t is not base else moved for t in (x, w, b)) for moved in (up, down)]
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(diff - float(grad.view(-1)[i])) <= tol


def test_norm_without_parameters_in_place_and_frozen(kt):
    gen = torch.Generator().manual_seed(4)
    for dtype, rows, cols in ((F32, 5, 100), (BF16, 6, 4096), (F32, 3, 8500)):
        x, dout = matrix(gen, rows, cols, dtype), matrix(gen, rows, cols, dtype)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        ones, zeros = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
        want = torch.empty_like(x)
        kt.kt_norm_forward(x, ones, zeros, want, mean, rstd)
        y = x.clone()
        kt.kt_norm_forward(y, None, None, y)                          # nothing kept, in place
        assert torch.equal(y, want)
        dx = torch.empty_like(x)
        work = torch.empty(kt.kt_norm_workspace(rows, cols), dtype=torch.uint8, device="cuda")
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        kt.kt_norm_backward(dout, ones, rstd, dx, dw, db, work, x=x, mean=mean)
        g = dout.clone()
        kt.kt_norm_backward(g, None, rstd, g, None, None, None, x=x, mean=mean)     # frozen, dx over dout
        assert torch.equal(g, dx)
        one = torch.full((cols,), math.nan, device="cuda")
        g = dout.clone()
        kt.kt_norm_backward(g, ones, rstd, g, None, one, work, x=x, mean=mean)      # dx over dout, bias alone
        assert torch.equal(one, db) and torch.equal(g, dx)


def test_norm_constant_rows_no_rows_and_repeats(kt):
    x = torch.full((4, 640), 3.0, device="cuda")
    out, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    kt.kt_norm_forward(x, None, None, out, mean, rstd, eps=1e-5)
    assert (mean == 3.0).all() and not out.any() and ((rstd - 1e-5 ** -0.5).abs() < 1e-4).all()
    none = torch.empty(0, 640, device="cuda")
    kt.kt_norm_forward(none, None, None, none, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"))
    dw, db = torch.full((640,), math.nan, device="cuda"), torch.full((640,), math.nan, device="cuda")
    kt.kt_norm_backward(none, None, torch.empty(0, device="cuda"), none, dw, db, None, x=none, mean=torch.empty(0, device="cuda"))
    assert not dw.any() and not db.any()                               # a sum over no rows
    gen = torch.Generator().manual_seed(5)
    x, dout = matrix(gen, 3000, 768, BF16), matrix(gen, 3000, 768, BF16)
    mean, rstd, out = torch.empty(3000, device="cuda"), torch.empty(3000, device="cuda"), torch.empty_like(x)
    kt.kt_norm_forward(x, None, None, out, mean, rstd)
    work = torch.empty(kt.kt_norm_workspace(3000, 768), dtype=torch.uint8, device="cuda")
    got = []
    for _ in range(3):
        dx, dw, db = torch.empty_like(x), torch.empty(768, device="cuda"), torch.empty(768, device="cuda")
        kt.kt_norm_backward(dout, None, rstd, dx, dw, db, work, x=x, mean=mean)
        got.append((dx, dw, db))
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


@pytest.mark.parametrize("layout", ["plain", "strided", "odd"])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_act(kt, rows, cols, dtype, kind, layout):
    gen = torch.Generator().manual_seed(rows * 31 + cols)
    x, dout = matrix(gen, rows, cols, dtype, layout, std=3.0), matrix(gen, rows, cols, dtype, layout)
    out = blank(x)
    codes, scales = checkpoint(kt, rows, cols)
    kt.kt_act_forward(x, out, codes, scales, kind)
    X = x.double()

    def gate_and_slope(v):
        if kind == "gelu":
            gate = torch.special.ndtr(v)
            return gate, gate + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        gate = torch.sigmoid(v)
        return gate, gate + v * gate * (1 - gate)

    # the normal distribution function: 0.75e-7 from the polynomial; exp and the quotients: 2^-22 each at arguments below 100
    e_gate = 0.75e-7 + 2.0 ** -20
    gate, _ = gate_and_slope(X)
    assert ((out.double() - X * gate).abs() <= X.abs() * e_gate + rounding(dtype) * (X * gate).abs()).all()
    assert surroundings_untouched(out)
    want_codes, want_scales = encode_exactly(x.float())
    assert torch.equal(codes[:, :cols].float(), want_codes) and torch.equal(scales, want_scales) and not codes[:, cols:].any()
    for kept in (True, False):
        dx = blank(x)
        kt.kt_act_backward(dout, codes if kept else None, scales if kept else None, dx, kind, x=None if kept else x)
        v = decode(codes, scales, cols) if kept else X
        _, slope = gate_and_slope(v)
        want = dout.double() * slope
        tol = dout.double().abs() * (e_gate * (2 + v.abs()) + 8 * U32 * (1 + v.abs())) + rounding(dtype) * want.abs()
        assert ((dx.double() - want).abs() <= tol).all()
        assert surroundings_untouched(dx)
    plain, in_place = blank(x), x.clone() if layout == "plain" else x
    kt.kt_act_forward(x, plain, kind=kind)                             # nothing kept
    assert torch.equal(plain, out)
    kt.kt_act_forward(in_place, in_place, kind=kind)
    assert torch.equal(in_place, out)


def test_act_against_differences(kt):
    """dx against central differences of the forward kernel: third derivatives below 2, outputs below 8
    off by at most 8 * 2^-19 (see test_act) over 2 h."""
    x = torch.linspace(-6, 6, 257, device="cuda").view(1, -1)
    h = 2.0 ** -5
    one = torch.ones_like(x)
    for kind in ("gelu", "silu"):
        dx, up, down = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        kt.kt_act_backward(one, None, None, dx, kind, x=x)
        kt.kt_act_forward(x + h, up, kind=kind)
        kt.kt_act_forward(x - h, down, kind=kind)
        assert ((up.double() - down.double()) / (2 * h) - dx.double()).abs().max() <= h * h / 6 * 2 + 8 * 2.0 ** -19 / h


@pytest.mark.parametrize("layout", ["plain", "strided", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_checkpoint(kt, rows, cols, dtype, layout):
    gen = torch.Generator().manual_seed(rows + cols)
    x = matrix(gen, rows, cols, dtype, layout)
    codes, scales = checkpoint(kt, rows, cols)
    kt.kt_ckpt_store(x, codes, scales)
    want_codes, want_scales = encode_exactly(x.float())
    assert torch.equal(codes[:, :cols].float(), want_codes) and torch.equal(scales, want_scales) and not codes[:, cols:].any()
    out = blank(x)
    kt.kt_ckpt_restore(codes, scales, out)
    at = torch.arange(cols, device="cuda") // 128
    value = codes[:, :cols].float() * scales[:, at]
    assert torch.equal(out, value.to(dtype)) and surroundings_untouched(out)
    step = scales.double()[:, at]
    assert ((value.double() - x.double()).abs() <= step * (0.5 + 127 * 4 * U32)).all()
    w, b = torch.randn(cols, generator=gen).cuda(), torch.randn(cols, generator=gen).cuda()
    kt.kt_ckpt_restore(codes, scales, out, w, b)
    want = value.double() * w.double() + b.double()
    assert ((out.double() - want).abs() <= rounding(dtype) * want.abs() + U32 * (2 * (value * w).abs() + b.abs())).all()


def test_checkpoint_of_extremes(kt):
    """Zeros, the smallest and the largest values, and blocks with an infinity or a NaN."""
    x = torch.zeros(6, 300, device="cuda")
    x[1] = 2.0 ** -101                                                   # below the smallest block that is kept
    x[2] = 2.0 ** -100
    x[3] = torch.finfo(F32).max
    x[3, ::2] *= -1
    x[4] = 1.0
    x[4, 130] = math.inf
    x[5] = 1.0
    x[5, 299] = math.nan
    codes, scales = checkpoint(kt, 6, 300)
    kt.kt_ckpt_store(x, codes, scales)
    back = torch.empty_like(x)
    kt.kt_ckpt_restore(codes, scales, back)
    assert not back[:2].any()
    assert ((back[2:4] / x[2:4] - 1).abs() <= 4 * U32).all()
    for r, bad in ((4, 1), (5, 2)):
        for blk in range(3):
            part = back[r, blk * 128:(blk + 1) * 128]
            assert torch.isnan(part).all() if blk == bad else ((part - 1).abs() <= 4 * U32).all()


def test_on_another_stream_and_recorded(kt):
    """A stream of the caller's own, and the same calls replayed from a stream capture."""
    gen = torch.Generator().manual_seed(6)
    x, dout = matrix(gen, 64, 1024, BF16), matrix(gen, 64, 1024, BF16)
    w, b = torch.randn(1024, generator=gen).cuda(), torch.randn(1024, generator=gen).cuda()

    def buffers():
        return [torch.zeros_like(x), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"), *checkpoint(kt, 64, 1024),
                torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b),
                torch.zeros(kt.kt_norm_workspace(64, 1024), dtype=torch.uint8, device="cuda")]

    def step(o, stream=None):
        kt.kt_norm_forward(x, w, b, o[0], o[1], o[2], 1e-5, o[3], o[4], stream=stream)
        kt.kt_norm_backward(dout, w, o[2], o[5], o[6], o[7], o[8], codes=o[3], scales=o[4], stream=stream)

    want, other, recorded = buffers(), buffers(), buffers()
    step(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(other, s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(recorded)
    graph.replay()
    torch.cuda.synchronize()
    for got in (other, recorded):
        assert all(torch.equal(a, c) for a, c in zip(got[:8], want[:8]))


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [300, 6000])
def test_sums_over_many_wide_rows(kt, rows, dtype, kept):
    """Rows of more than 8192 columns: dweight and dbias of one 2^24 and then ones, of which a sum that takes one row after the
    other loses every one.  A column passes through 64 additions in a block of rows, one for each of its range's two
    blocks, and 12 over the partial sums: 80 of them at most, each off by at most u32 of all terms."""
    cols = 8200
    dout = torch.ones(rows, cols, dtype=dtype, device="cuda")
    dout[0] = 2.0 ** 24
    ones = torch.ones(rows, device="cuda")
    if kept:
        codes, scales = checkpoint(kt, rows, cols)
        source = {"codes": codes.fill_(1), "scales": scales.fill_(1.0)}
    else:
        source = {"x": torch.ones_like(dout), "mean": torch.zeros_like(ones)}
    dx, dw, db = torch.empty_like(dout), torch.full((cols,), math.nan, device="cuda"), torch.full((cols,), math.nan, device="cuda")
    work = torch.full((kt.kt_norm_workspace(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    kt.kt_norm_backward(dout, None, ones, dx, dw, db, work, **source)
    want = 2.0 ** 24 + rows - 1
    for got in (dw, db):
        assert ((got.double() - want).abs() <= 80 * U32 * want).all()


def test_gelu_of_fp32_rows(kt):
    """fp32 rows get the normal tail T(a) = Phi(-a) to fp32 as well.

    In units of u32: T comes from a reciprocal and a polynomial of nine terms (24 at most) and an exponential (4) of a^2 / 2,
    whose three roundings are 1.5 a^2 of it: 32 + 2 a^2 of T; the density's share a phi is off by 8 + 2 a^2 of itself.
    Below 1 in magnitude Phi is a polynomial in x^2 around 1/2, off by 3 in all.  Above 1, 1 - T is rounded once; below -1
    nothing is: there the tolerance falls with the value."""
    gen = torch.Generator().manual_seed(17)
    x = torch.cat([torch.linspace(-12, 12, 24 * 1024 + 1), torch.randn(65535, generator=gen) * 2]).cuda().view(2, -1)
    dout = torch.randn(x.shape, generator=gen).cuda()
    out, dx = torch.empty_like(x), torch.empty_like(x)
    kt.kt_act_forward(x, out, kind="gelu")
    kt.kt_act_backward(dout, None, None, dx, "gelu", x=x)
    X, D = x.double(), dout.double()
    A = X.abs()

    def normal(v):                                   # torch's ndtr is (1 + erf) / 2, which has no tail
        return torch.special.erfc(-v / math.sqrt(2)) / 2

    T, phi = normal(-A), torch.exp(-A * A / 2) / math.sqrt(2 * math.pi)
    e_tail = T * (32 + 2 * A * A)
    want = X * normal(X)
    tol = U32 * (torch.where(A < 1, 4 * A, A * e_tail) + 2 * want.abs())
    assert ((out.double() - want).abs() <= tol + 2.0 ** -126).all()
    want = D * (normal(X) + X * phi)
    tol = U32 * (D.abs() * (torch.where(A < 1, 4.0, torch.where(X > 0, 2.0, 0.0) + e_tail) + A * phi * (8 + 2 * A * A)) + 2 * want.abs())
    assert ((dx.double() - want).abs() <= tol + D.abs() * 2.0 ** -120).all()
    edge = torch.tensor([[0.0, -0.0, math.inf, -math.inf, math.nan, 3e38, -3e38, 1e-40]], device="cuda")
    out, dx = torch.empty_like(edge), torch.empty_like(edge)
    kt.kt_act_forward(edge, out, kind="gelu")
    kt.kt_act_backward(torch.ones_like(edge), None, None, dx, "gelu", x=edge)
    assert torch.equal(out[0, [0, 1, 2, 3, 5, 6]].abs(), torch.tensor([0.0, 0.0, math.inf, 0.0, 3e38, 0.0], device="cuda")) and torch.isnan(out[0, 4])
    assert torch.equal(dx[0, [0, 1, 2, 3, 5, 6, 7]], torch.tensor([0.5, 0.5, 1.0, 0.0, 1.0, 0.0, 0.5], device="cuda")) and torch.isnan(dx[0, 4])


@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols,group", [(72, 32), (250, 32), (500, 32), (1000, 64), (1500, 96), (2000, 128), (2500, 160), (3000, 192), (4000, 256), (5000, 320),
                                        (6000, 384), (8000, 512)])
def test_norm_with_rows_ahead(kt, cols, group, dtype, layout):
    """At least six rows to every group of threads (of which an SM holds 768 / group): the places of the rows that are copied ahead, three or
    four of them, are filled a second time, and all of it is compared."""
    test_norm(kt, 6 * 148 * (768 // group), cols, dtype, F32, layout)


def in_parts(kt, call, rows, cols, dtype, parts):
    """What `call` makes of a matrix in one call and in several calls on parts of its rows: the same bits."""
    gen = torch.Generator("cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=gen, dtype=dtype, device="cuda")
    got = []
    for pieces in (1, parts):
        out = [torch.full_like(x, math.nan), *checkpoint(kt, rows, cols), torch.full_like(x, math.nan)]
        for k in range(pieces):
            mine = slice(rows * k // pieces, rows * (k + 1) // pieces)
            call(x[mine], *(o[mine] for o in out))
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert not torch.isnan(got[0][0]).any() and not torch.isnan(got[0][3]).any()


@pytest.mark.parametrize("dtype,rows,cols", [(BF16, 1030, 1 << 17), (BF16, (1 << 26) + 3, 8), (BF16, (1 << 26) + 3, 1), (F32, (1 << 25) + 3, 4)])
def test_activations_in_more_than_one_piece(kt, dtype, rows, cols):
    """Sizes that one call goes through in two pieces: 2^27 elements of a gapless matrix, 2^30 vectors (of rows padded to whole
    blocks) of another, by vectors and by elements."""
    def call(x, out, codes, scales, dx):
        kt.kt_act_forward(x, out, codes, scales, "gelu")
        kt.kt_act_backward(x, codes, scales, dx, "gelu")

    in_parts(kt, call, rows, cols, dtype, 5)

    def restore(x, out, codes, scales, dx):
        kt.kt_ckpt_store(x, codes, scales)
        kt.kt_ckpt_restore(codes, scales, out)
        kt.kt_act_backward(x, None, None, dx, "silu", x=x)

    in_parts(kt, restore, rows, cols, dtype, 5)
