"""Attention and its gradients against the formulas in 64 bits, on the GPU.

Tolerances are derived, element by element.  Products of bf16 are exact and summed in fp32: a sum over D
terms is off by at most (D + 8) 2^-23 sum |terms| (the tensor cores may cut instead of round).  That error
of a score is a relative error of its probability, to which the exponential adds 2^-20 (its own 2^-22, the
argument's rounding).  Probabilities and dS are rounded to bf16 (2^-8: it keeps 8 significant bits) before the second product, results
again.  A sum over n tokens adds n 2^-23 of its absolute terms.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
U23, U8 = 2.0 ** -23, 2.0 ** -8


@pytest.fixture(scope="module")
def kt():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import binding
    torch.cuda.set_device(0)
    yield binding
    assert binding.kt_attn_given_up() == 0


def heads(gen, B, L, H, D, layout, fill=None):
    """[B, L, H, D] of bf16: tokens first, heads first, one of three in a shared buffer, or with gaps."""
    x = (torch.randn(B, L, H, D, generator=gen) if fill is None else torch.full((B, L, H, D), fill)).to(BF16)
    if layout == "heads first":
        t = torch.empty(B, H, L, D, dtype=BF16, device="cuda").transpose(1, 2)
    elif layout == "one of three":
        t = torch.empty(B, L, 3, H, D, dtype=BF16, device="cuda")[:, :, 1]
    elif layout == "gaps":
        t = torch.full((B, L + 3, H, D + 24), math.nan, dtype=BF16, device="cuda")[:, 2:L + 2, :, 8:D + 8]
    else:
        t = torch.empty(B, L, H, D, dtype=BF16, device="cuda")
    t.copy_(x)
    return t


def mask_of(B, Lq, Lk, causal, used_q, used_kv):
    n = torch.full((B,), Lq) if used_q is None else torch.tensor(used_q).clamp(0, Lq)
    m = torch.full((B,), Lk) if used_kv is None else torch.tensor(used_kv).clamp(0, Lk)
    i, j = torch.arange(Lq)[None, :, None], torch.arange(Lk)[None, None, :]
    seen = (i < n[:, None, None]) & (j < m[:, None, None])
    if causal:
        seen &= j <= i + (m - n)[:, None, None]
    return seen[:, None].cuda(), n, m


def wide(x, H):
    return x.double().transpose(1, 2).repeat_interleave(H // x.shape[2], 1)


def check(got, want, tol, what):
    bad = ~((got - want).abs() <= tol)          # NaN is bad
    assert not bad.any(), "%s: %d of %d off, worst %.3g where %.3g is allowed" % (
        what, int(bad.sum()), bad.numel(), float((got - want).abs()[bad].nan_to_num(nan=math.inf).max()), float(tol[bad].min()))


def run_case(kt, B, Lq, Lk, H, Hk, D, causal=False, used_q=None, used_kv=None, layout="plain", scale=None, seed=0, stream=None):
    gen = torch.Generator().manual_seed(seed)
    q, k, v, dout = heads(gen, B, Lq, H, D, layout), heads(gen, B, Lk, Hk, D, layout), heads(gen, B, Lk, Hk, D, layout), heads(gen, B, Lq, H, D, layout)
    seen, n, m = mask_of(B, Lq, Lk, causal, used_q, used_kv)
    clean = [t.clone() for t in (q, k, v, dout)]
    for b in range(B):                           # what lies past the tokens in use does not matter
        for t, c, u in ((q, clean[0], n), (dout, clean[3], n), (k, clean[1], m), (v, clean[2], m)):
            t[b, int(u[b]):] = math.nan
            t[b, int(u[b])::2] = math.inf
            c[b, int(u[b]):] = 0
    uq, uk = (None if u is None else torch.tensor(u, dtype=torch.int32, device="cuda") for u in (used_q, used_kv))
    out, lse = heads(gen, B, Lq, H, D, layout, math.nan), torch.full((B, H, Lq), math.nan, device="cuda")
    mask = {"scale": scale, "causal": causal, "used_q": uq, "used_kv": uk, "stream": stream}
    kt.kt_attn_forward(q, k, v, out, lse, **mask)
    scale = D ** -0.5 if scale is None else scale
    Q, K, V, G = (wide(t, H) for t in clean)
    S = (Q @ K.transpose(2, 3)) * scale
    e_s = (D + 8) * U23 * scale * (Q.abs() @ K.abs().transpose(2, 3))     # error of a score
    S = S.masked_fill(~seen, -math.inf)
    L = torch.logsumexp(S, 3) if Lk else torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device="cuda")
    P = torch.exp(S - L[..., None]).nan_to_num(nan=0.0)
    e_row = (e_s * seen).amax(3) if Lk else torch.zeros_like(L)
    if stream is not None:
        stream.synchronize()
    empty = L == -math.inf
    assert torch.equal(lse.double() == -math.inf, empty)
    check(lse.double().masked_fill(empty, 0), L.masked_fill(empty, 0), e_row + 2.0 ** -20 * (1 + L.masked_fill(empty, 0).abs()) + (Lk + 8) * U23, "lse")
    e_p = 2 * e_row[..., None] + 2.0 ** -19 + 2 * (Lk + 8) * U23
    O = P @ V
    check(out.double().transpose(1, 2), O, (P @ V.abs()) * (U8 + e_p) * 1.01 + U8 * O.abs(), "out")
    assert not out[~seen.any(3).expand(B, H, Lq).transpose(1, 2)].any()

    dq, dk, dv = heads(gen, B, Lq, H, D, layout, math.nan), heads(gen, B, Lk, Hk, D, layout, math.nan), heads(gen, B, Lk, Hk, D, layout, math.nan)
    for b in range(B):                           # nor what the saved tensors hold there
        out[b, int(n[b]):] = math.nan
        lse[b, :, int(n[b]):] = math.nan
    work = torch.full((max(1, kt.kt_attn_workspace(q, k)),), 255, dtype=torch.uint8, device="cuda")
    kt.kt_attn_backward(dout, q, k, v, out, lse, dq, dk, dv, work, **mask)
    if stream is not None:
        stream.synchronize()
    used = torch.arange(Lq)[None, :] < n[:, None]
    saved = torch.where(used.cuda()[:, None, :, None], wide(out, H), 0.0)
    E = torch.where(used.cuda()[:, None], lse.double(), -math.inf)
    P = torch.exp(S - E[..., None]).nan_to_num(nan=0.0).masked_fill(~seen, 0)
    e_p = e_s + 2.0 ** -19
    delta = (G * saved).sum(3, keepdim=True)
    dP = G @ V.transpose(2, 3)
    dS = P * (dP - delta)
    e_ds = dS.abs() * (U8 + e_p) * 1.01 + P * (D + 8) * U23 * (G.abs() @ V.abs().transpose(2, 3) + (G.abs() * saved.abs()).sum(3, keepdim=True))

    def shared(x):                               # heads that share keys are summed
        return x.view(B, Hk, H // Hk, Lk, D).sum(2)

    want, tol = dS @ K * scale, (e_ds @ K.abs() + Lk * U23 * (dS.abs() @ K.abs())) * scale
    check(dq.double().transpose(1, 2), want, tol * 1.01 + U8 * want.abs() + 1e-30, "dq")
    dSt, Pt = dS.transpose(2, 3), P.transpose(2, 3)
    nq = Lq * (H // Hk)
    want, tol = shared(dSt @ Q) * scale, shared(e_ds.transpose(2, 3) @ Q.abs() + nq * U23 * (dSt.abs() @ Q.abs())) * scale
    check(dk.double().transpose(1, 2), want, tol * 1.01 + U8 * want.abs() + 1e-30, "dk")
    want, tol = shared(Pt @ G), shared((Pt * (U8 + e_p.transpose(2, 3) + nq * U23)) @ G.abs())
    check(dv.double().transpose(1, 2), want, tol * 1.01 + U8 * want.abs() + 1e-30, "dv")
    for b in range(B):
        assert not dq[b, int(n[b]):].any() and not dk[b, int(m[b]):].any() and not dv[b, int(m[b]):].any()
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 5), (7, 1), (127, 128), (128, 127), (129, 130), (256, 256), (300, 200), (200, 300), (513, 700)])
def test_lengths(kt, Lq, Lk, dim, causal):
    run_case(kt, 2, Lq, Lk, 2, 1, dim, causal, seed=Lq * 1000 + Lk + dim)


@pytest.mark.parametrize("dim", [8, 16, 40, 56, 72, 80, 96, 120])
def test_head_sizes(kt, dim):
    run_case(kt, 1, 150, 170, 3, 3, dim, True, seed=dim)


@pytest.mark.parametrize("H,Hk", [(1, 1), (8, 8), (8, 2), (6, 1), (15, 5)])
def test_shared_heads(kt, H, Hk):
    run_case(kt, 2, 190, 260, H, Hk, 64, True, seed=H * 16 + Hk)


@pytest.mark.parametrize("layout", ["heads first", "one of three", "gaps"])
@pytest.mark.parametrize("dim", [64, 104])
def test_layouts(kt, layout, dim):
    run_case(kt, 2, 140, 140, 4, 4, dim, True, layout=layout, seed=dim)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("used_q,used_kv", [([300, 1, 0, 257], [300, 1, 0, 257]), ([128, 300, 5, 129], [1, 0, 300, 128]), (None, [0, 0, 0, 0]),
                                            ([0, 0, 0, 0], None), ([299, 130, 200, 64], None), (None, [400, 299, -3, 100])])
def test_sequences_of_different_lengths(kt, used_q, used_kv, dim, causal):
    run_case(kt, 4, 300, 300, 4, 2, dim, causal, used_q, used_kv, seed=7)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [48, 128])
@pytest.mark.parametrize("Lq,Lk,H,Hk", [(1, 1100, 2, 1), (1, 4100, 20, 5), (5, 2049, 4, 4), (260, 1500, 3, 1), (900, 1024, 12, 12)])
def test_few_long_rows(kt, Lq, Lk, H, Hk, dim, causal):
    """Fewer query tiles than SMs: several CTAs share the keys of one (2, 4 and 8 at these sizes)."""
    run_case(kt, 2, Lq, Lk, H, Hk, dim, causal, seed=Lq + Lk)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 112])
@pytest.mark.parametrize("Lq,Lk,H,Hk,used_q,used_kv", [(700, 700, 8, 1, None, None), (1500, 300, 2, 2, None, None), (400, 140, 12, 2, [400, 0], None), (1300, 1300, 3, 1, [7, 1200], [1300, 129]), (1400, 1400, 8, 2, None, [1400, 900])])
def test_few_long_columns(kt, Lq, Lk, H, Hk, used_q, used_kv, dim, causal):
    """Few key tiles that many query tiles see: several CTAs share the queries of one in the backward pass (2, 4 and 8 at these sizes)."""
    run_case(kt, 2, Lq, Lk, H, Hk, dim, causal, used_q, used_kv, seed=Lq + H)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("used_q,used_kv", [([3, 1, 0, 3], [2000, 1, 700, 0]), (None, [129, 0, 2000, 128]), ([3, 2, 1, 3], None)])
def test_few_long_rows_of_different_lengths(kt, used_q, used_kv, dim):
    for causal in (False, True):
        run_case(kt, 4, 3, 2000, 2, 2, dim, causal, used_q, used_kv, layout="gaps", seed=dim)


@pytest.mark.parametrize("Lq,Lk", [(5, 0), (0, 5), (0, 0)])
def test_no_tokens(kt, Lq, Lk):
    q, kv = torch.ones(2, Lq, 2, 64, dtype=BF16, device="cuda"), torch.ones(2, Lk, 2, 64, dtype=BF16, device="cuda")
    out, lse = torch.full_like(q, math.nan), torch.full((2, 2, Lq), math.nan, device="cuda")
    kt.kt_attn_forward(q, kv, kv, out, lse)
    assert not out.any() and (lse == -math.inf).all()
    dq, dk, dv = torch.full_like(q, math.nan), torch.full_like(kv, math.nan), torch.full_like(kv, math.nan)
    kt.kt_attn_backward(q, q, kv, kv, out, lse, dq, dk, dv, torch.empty(max(1, kt.kt_attn_workspace(q, kv)), dtype=torch.uint8, device="cuda"))
    assert not dq.any() and not dk.any() and not dv.any()


def test_large_scores_and_scales(kt):
    """Scores of some hundreds: the running maximum jumps from tile to tile; and nearly even probabilities."""
    run_case(kt, 1, 260, 520, 2, 2, 64, False, scale=12.0, seed=11)
    run_case(kt, 1, 260, 520, 2, 2, 128, True, scale=1e-4, seed=12)


def test_growing_scores(kt):
    """Keys whose scores grow from tile to tile by more than the probabilities' range."""
    q = torch.ones(1, 128, 1, 64, dtype=BF16, device="cuda")
    k = (torch.arange(640, device="cuda").view(1, 640, 1, 1) // 64 * 0.25).expand(1, 640, 1, 64).to(BF16).contiguous()
    v = torch.randn(1, 640, 1, 64, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    out, lse = torch.empty_like(q), torch.empty(1, 1, 128, device="cuda")
    kt.kt_attn_forward(q, k, v, out, lse, scale=1.0)
    S = wide(q, 1) @ wide(k, 1).transpose(2, 3)                   # 0, 16, 32 ... 144: exact
    P = torch.softmax(S, 3)
    check(lse.double(), torch.logsumexp(S, 3), torch.full_like(lse.double(), 2.0 ** -20 * 150), "lse")
    check(out.double().transpose(1, 2), P @ wide(v, 1), (P @ wide(v, 1).abs()) * (2 * U8 + 2.0 ** -17), "out")


def test_a_not_a_number_in_use_reaches_its_results(kt):
    gen = torch.Generator().manual_seed(9)
    q, k, v = (heads(gen, 1, 200, 1, 64, "plain") for _ in range(3))
    q[0, 150, 0, 3] = math.nan
    out, lse = torch.empty_like(q), torch.empty(1, 1, 200, device="cuda")
    kt.kt_attn_forward(q, k, v, out, lse)
    rows = torch.isnan(out[0, :, 0]).all(1)
    assert rows[150] and int(rows.sum()) == 1 and torch.isnan(lse[0, 0, 150]) and not torch.isnan(out[0, :150]).any()


@pytest.mark.parametrize("dim", [64, 128])
def test_long(kt, dim):
    run_case(kt, 1, 2500, 2500, 2, 1, dim, True, seed=3)


def test_many_heads_fill_the_device(kt):
    run_case(kt, 7, 180, 180, 48, 16, 64, True, seed=4)


def test_against_differences(kt):
    """Gradients against central differences of the definition in 64 bits along random directions: what the
    definition itself allows (h^2) and what bf16 results allow (2^-8 of the absolute sum)."""
    gen = torch.Generator().manual_seed(21)
    B, L, H, Hk, D = 1, 37, 2, 1, 16
    q, k, v, dout = heads(gen, B, L, H, D, "plain"), heads(gen, B, L, Hk, D, "plain"), heads(gen, B, L, Hk, D, "plain"), heads(gen, B, L, H, D, "plain")
    out, lse = torch.empty_like(q), torch.empty(B, H, L, device="cuda")
    kt.kt_attn_forward(q, k, v, out, lse, causal=True)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    kt.kt_attn_backward(dout, q, k, v, out, lse, *grads, torch.empty(kt.kt_attn_workspace(q, k), dtype=torch.uint8, device="cuda"), causal=True)
    seen, _, _ = mask_of(B, L, L, True, None, None)

    def loss(ts):
        Q, K, V = (wide(t, H) for t in ts)
        S = (Q @ K.transpose(2, 3) / math.sqrt(D)).masked_fill(~seen, -math.inf)
        return float((torch.softmax(S, 3) @ V * wide(dout, H)).sum())

    h = 1e-4
    for which in range(3):
        for _ in range(4):
            step = torch.randn(grads[which].shape, generator=gen, dtype=torch.float64).cuda()
            ts = [t.double() for t in (q, k, v)]
            up, down = list(ts), list(ts)
            up[which], down[which] = ts[which] + h * step, ts[which] - h * step
            diff = (loss(up) - loss(down)) / (2 * h)
            # every gradient is within 2^-8 of itself and of the absolute terms of its sum: a few times its size
            assert abs(diff - float((grads[which].double() * step).sum())) <= 2.0 ** -7 * float((grads[which].double() * step).abs().sum()) + 1e-3


def test_repeats_streams_and_recordings(kt):
    gen = torch.Generator().manual_seed(31)
    q, k, v, dout = (heads(gen, 2, 333, 4, 80, "plain") for _ in range(4))
    work = torch.empty(kt.kt_attn_workspace(q, k), dtype=torch.uint8, device="cuda")

    def buffers():
        return [torch.zeros_like(q), torch.zeros(2, 4, 333, device="cuda"), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]

    def step(o, stream=None):
        kt.kt_attn_forward(q, k, v, o[0], o[1], causal=True, stream=stream)
        kt.kt_attn_backward(dout, q, k, v, o[0], o[1], *o[2:], work, causal=True, stream=stream)

    want, again, other, recorded = buffers(), buffers(), buffers(), buffers()
    step(want)
    step(again)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(other, s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(recorded)
    graph.replay()
    torch.cuda.synchronize()
    for got in (again, other, recorded):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refused(kt):
    q, k = torch.zeros(2, 16, 4, 64, dtype=BF16, device="cuda"), torch.zeros(2, 16, 2, 64, dtype=BF16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(2, 4, 16, device="cuda")

    def status(*args, **kw):
        with pytest.raises(kt.KtError) as e:
            kt.kt_attn_forward(*args, **kw)
        return e.value.status

    assert status(q.float(), k, k, out, lse) == kt.KT_ERR_SHAPE
    assert status(q, k, k[:, :8], out, lse) == kt.KT_ERR_SHAPE
    assert status(q, k, k, out, lse.double()) == kt.KT_ERR_SHAPE
    assert status(q, k, k, out, lse[:, :, :8]) == kt.KT_ERR_SHAPE
    assert status(q[:, :, :3], k, k, out[:, :, :3], lse[:, :3].contiguous()) == kt.KT_ERR_SHAPE           # 3 heads cannot share 2
    assert status(q, k, k, out, lse, scale=0.0) == kt.KT_ERR_INVALID
    assert status(q, k, k, out, lse, scale=math.nan) == kt.KT_ERR_INVALID
    assert status(q, k, k, out, lse, used_q=torch.zeros(2, device="cuda")) == kt.KT_ERR_SHAPE
    assert status(q[..., :60], k[..., :60], k[..., :60], out[..., :60], lse) == kt.KT_ERR_SHAPE          # head_dim 60
    assert status(q[..., 4:60], k[..., 4:60], k[..., 4:60], out[..., 4:60], lse) == kt.KT_ERR_ALIGN      # 8 bytes into a vector
    wide_q = torch.zeros(2, 16, 4, 136, dtype=BF16, device="cuda")
    assert status(wide_q, wide_q, wide_q, wide_q, lse) == kt.KT_ERR_SHAPE
    assert status(q, k[:, :1].expand(2, 16, 2, 64), k, out, lse) == kt.KT_ERR_SHAPE                      # stride 0
    work = torch.empty(kt.kt_attn_workspace(q, k) - 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(kt.KtError) as e:
        kt.kt_attn_backward(q, q, k, k, out, lse, torch.empty_like(q), torch.empty_like(k), torch.empty_like(k), work)
    assert e.value.status == kt.KT_ERR_SHAPE


@pytest.mark.parametrize("Lq,Lk,H,Hk,causal", [(2100, 2100, 4, 1, True), (3000, 900, 6, 2, False)])
def test_many_query_tiles_to_a_key_tile(kt, Lq, Lk, H, Hk, causal):
    """Heads of 128: dP of a query tile takes the place of the last one's P and dS. Dozens of tiles in a row, against the
    formulas, and the same bits every time while another stream keeps the device busy."""
    want = run_case(kt, 1, Lq, Lk, H, Hk, 128, causal, seed=Lq)
    s = torch.cuda.Stream()
    for i in range(4):
        with torch.cuda.stream(s):
            a = torch.randn(2048, 2048, device="cuda", dtype=BF16)
            for _ in range(i):
                a = a @ a * 0.01
        got = run_case(kt, 1, Lq, Lk, H, Hk, 128, causal, seed=Lq)
        assert all(torch.equal(x.nan_to_num(nan=0.0), y.nan_to_num(nan=0.0)) for x, y in zip(got, want))
