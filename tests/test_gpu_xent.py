"""Cross entropy over a vocabulary and its gradient against their formulas in 64 bits, on the GPU.

Tolerances are derived.  A logit is a sum of dim products of bf16 (exact in fp32) added in fp32, 16 at a time: off by at
most (dim / 16 + 16) * 2^-23 * size with size = scale * sum |h| |w| (the tensor cores cut off where fp32 rounds, hence
2^-23).  That is the error of a maximum and of a target's logit, and of lse; the exponentials add 2^-22 each, a sum
of them (256 columns, the joined tiles) at most 400 * 2^-24, the logarithm 2^-23 of its value.

P = scale (g + z) exp(l - lse) - scale g [target] is off by the logit's error and 2^-21 relative to its first term, and
by half a step of bf16, 2^-8, relative to itself (it is rounded in units of its row: the same relative to itself); where
the rows' units differ, dW is formed from hidden rows times their units, rounded to bf16: 2^-8 of P's size times |h| more.  The products with W and h add those errors times |W| and |h|, sums in fp32
((terms / 16 + 64) * 2^-23 of the terms' sizes), and the result half a step, 2^-8.  What is below fp32's and bf16's smallest
normal number, 2^-126, may become zero wherever it appears: an exponential (so P is off by scale |g + z| 2^-126 more), P itself,
each of the terms and the result."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U16, TINY = 2.0 ** -8, 2.0 ** -126
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def kt():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import binding
    torch.cuda.set_device(0)
    return binding


def strided(x, pad):
    """x with rows `pad` elements further apart, NaN between them."""
    if pad == 0:
        return x.cuda()
    buf = torch.full((x.size(0), x.size(1) + pad), float("nan"), dtype=x.dtype, device="cuda")
    buf[:, :x.size(1)] = x.cuda()
    return buf[:, :x.size(1)]


class Problem:
    def __init__(self, rows, dim, vocab, ignored=0.0, scale=1.0, pad=0, seed=0, std=1.0):
        gen = torch.Generator().manual_seed(seed + rows + dim + vocab)
        self.rows, self.dim, self.vocab, self.scale = rows, dim, vocab, scale
        self.hidden = strided((torch.randn(rows, dim, generator=gen) * std).to(BF16), pad)
        self.weight = strided((torch.randn(vocab, dim, generator=gen) * 2.0 * dim ** -0.5).to(BF16), pad)
        self.targets = torch.randint(vocab, (rows,), generator=gen)
        self.targets[torch.rand(rows, generator=gen) < ignored] = -100
        self.targets = self.targets.cuda()
        self.dloss, self.dlse = (torch.randn(rows, generator=gen).cuda() for _ in range(2))
        self.pad = pad

    def work(self, kt, backward):
        return torch.full((kt.kt_xent_workspace(self.rows, self.dim, self.vocab, backward),), 255, dtype=torch.uint8, device="cuda")

    def forward(self, kt):
        loss, lse = (torch.full((self.rows,), 5.0, device="cuda") for _ in range(2))
        kt.kt_xent_forward(self.hidden, self.weight, self.targets, loss, lse, self.work(kt, False), scale=self.scale)
        return loss, lse

    def backward(self, kt, lse, dlse=None, hidden=True, weight=True):
        dh = strided(torch.full((self.rows, self.dim), 3.0, dtype=BF16), self.pad) if hidden else None
        dw = strided(torch.full((self.vocab, self.dim), 3.0, dtype=BF16), self.pad) if weight else None
        kt.kt_xent_backward(self.dloss, self.hidden, self.weight, self.targets, lse, dh, dw, self.work(kt, True), scale=self.scale, dlse=dlse)
        return dh, dw

    def exact(self):
        """Logits, their errors' bound, lse, loss and which rows count, in 64 bits."""
        used = self.targets >= 0
        h, w = torch.where(used[:, None], self.hidden.double(), 0.0), self.weight.double()
        logits, sizes = self.scale * (h @ w.t()), self.scale * (h.abs() @ w.abs().t())
        lse = torch.logsumexp(logits, 1)
        loss = lse - logits.gather(1, self.targets.clamp(min=0)[:, None])[:, 0]
        off = (self.dim / 16 + 16) * 2.0 ** -23 * sizes
        return h, w, logits, off, torch.where(used, lse, 0.0), torch.where(used, loss, 0.0), used

    def check_forward(self, kt):
        loss, lse = self.forward(kt)
        _, _, _, off, want_lse, want_loss, used = self.exact()
        slack = off.amax(1) + 2.0 ** -22 + 400 * 2.0 ** -24 + 2.0 ** -22 * want_lse.abs()
        assert ((lse.double() - want_lse).abs() <= slack).all()
        assert ((loss.double() - want_loss).abs() <= 2 * slack).all()
        assert (loss[~used] == 0).all() and (lse[~used] == 0).all()
        return lse

    def check_backward(self, kt, lse, dlse=None, hidden=True, weight=True):
        dh, dw = self.backward(kt, lse, dlse, hidden, weight)
        h, w, logits, off, _, _, used = self.exact()
        g = torch.where(used, self.dloss.double(), 0.0)
        z = g if dlse is None else g + torch.where(used, dlse.double(), 0.0)
        p = torch.exp(logits - lse.double()[:, None]) * (self.scale * z)[:, None]
        p = torch.where(used[:, None], p, 0.0)
        del logits
        # (lse is rounded too: 2^-24 of its value, as is its product with log2(e))
        loose = p.abs() * (off + 2.0 ** -21 + 2.0 ** -22 * lse.double().abs()[:, None])
        p[torch.arange(self.rows, device="cuda"), self.targets.clamp(min=0)] -= self.scale * g
        loose += U16 * p.abs() + TINY * (1 + self.scale * z.abs())[:, None]
        if hidden:
            want = p @ w
            slack = loose @ w.abs() + (self.vocab / 16 + 64) * 2.0 ** -23 * (p.abs() @ w.abs()) + TINY * (self.vocab + 1)
            assert ((dh.double() - want).abs() <= slack + U16 * (want.abs() + slack)).all()
            assert (dh[~used] == 0).all()
        if weight:
            want = p.t() @ h
            slack = (loose + U16 * p.abs()).t() @ h.abs() + (self.rows / 16 + 64) * 2.0 ** -23 * (p.abs().t() @ h.abs()) + TINY * (self.rows + 1)
            assert ((dw.double() - want).abs() <= slack + U16 * (want.abs() + slack)).all()
        return dh, dw


SIZES = [(1, 8, 1), (1, 8, 2), (1, 64, 1000), (3, 16, 5), (63, 72, 127), (64, 64, 128), (65, 128, 129), (127, 200, 333), (128, 256, 256), (129, 320, 257), (300, 96, 8001), (24, 512, 32000),
         (1000, 136, 5003)]


@pytest.mark.parametrize("rows,dim,vocab", SIZES)
def test_one_cta_to_a_tile(kt, rows, dim, vocab):
    p = Problem(rows, dim, vocab)
    p.check_backward(kt, p.check_forward(kt))


@pytest.mark.parametrize("rows,dim,vocab,ignored,scale,pad", [(2500, 64, 5003, 0.0, 1.0, 0), (4096, 256, 2048, 0.3, 0.5, 8), (5000, 1032, 3001, 0.02, 2.0, 0), (257, 4096, 20000, 0.0, 1.0, 24), (3000, 2056, 12345, 0.6, 1.0, 8)])
def test_pairs_of_ctas(kt, rows, dim, vocab, ignored, scale, pad):
    p = Problem(rows, dim, vocab, ignored, scale, pad)
    p.check_backward(kt, p.check_forward(kt), dlse=p.dlse)


@pytest.mark.parametrize("rows,dim,vocab", [(200, 136, 1000), (1300, 64, 1000), (5, 64, 300)])
@pytest.mark.parametrize("ignored", [0.05, 0.5, 0.95, 1.1])
def test_rows_that_do_not_count(kt, rows, dim, vocab, ignored):
    """What hidden holds in them does not matter, and dweight is zeros where none counts."""
    p = Problem(rows, dim, vocab, ignored)
    if ignored < 1:
        p.targets[rows // 2] = 1
    used = p.targets >= 0
    p.hidden[~used] = float("nan")
    p.dloss[~used], p.dlse[~used] = float("nan"), float("inf")
    dh, dw = p.check_backward(kt, p.check_forward(kt), dlse=p.dlse)
    if ignored > 1:
        assert (dw == 0).all() and (dh == 0).all()


@pytest.mark.parametrize("rows,dim,vocab,ignored", [(5, 64, 300, 0.0), (200, 136, 1000, 0.3), (3000, 200, 5003, 0.1), (4096, 128, 2048, 0.0)])
@pytest.mark.parametrize("kind", ["mean", "weighted", "some zero", "zero", "only lse"])
def test_gradients_of_the_rows(kt, rows, dim, vocab, ignored, kind):
    """Rows that share a gradient (a mean's 1 / n, far from a power of two), that differ, that are zero; lse alone."""
    p = Problem(rows, dim, vocab, ignored)
    lse = p.check_forward(kt)
    p.dloss = {"mean": torch.full_like(p.dloss, 1.0 / 3891), "weighted": p.dloss * 1e-3, "some zero": p.dloss * (torch.arange(rows, device="cuda") % 3 > 0),
               "zero": torch.zeros_like(p.dloss), "only lse": torch.zeros_like(p.dloss)}[kind]
    dh, dw = p.check_backward(kt, lse, dlse=p.dlse if kind == "only lse" else None)
    if kind == "zero":
        assert (dh == 0).all() and (dw == 0).all()
    if kind == "mean" and dim == 200:
        # nearly all of a row is its target's entry, which the unit makes exact: the results' own rounding (2^-8 / sqrt(12) to
        # 2^-9 / sqrt(12), some 0.17 % rms) and hardly more
        h, w, logits, _, _, _, used = p.exact()
        q = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))
        q[torch.arange(rows, device="cuda"), p.targets.clamp(min=0)] -= 1.0
        q = torch.where(used[:, None], q * p.dloss.double()[:, None], 0.0)
        for got, want in ((dh, q @ w), (dw, q.t() @ h)):
            assert (got.double() - want).norm() <= 0.0022 * want.norm()


@pytest.mark.parametrize("hidden,weight", [(True, False), (False, True)])
def test_one_gradient_alone(kt, hidden, weight):
    p = Problem(300, 200, 3000, 0.1)
    lse = p.check_forward(kt)
    both = p.backward(kt, lse)
    one = p.check_backward(kt, lse, hidden=hidden, weight=weight)
    assert torch.equal(one[0] if hidden else one[1], both[0] if hidden else both[1])


def test_several_pieces_of_the_vocabulary(kt):
    """More columns than a piece takes at 8192 rows (32768): the last piece is 300 columns, fewer than any other."""
    p = Problem(8192, 16, 2 * 32768 + 300, 0.0)
    loss, lse = p.forward(kt)
    dh, dw = p.backward(kt, lse)
    some = torch.arange(5, 8192, 700, device="cuda")
    part = Problem(1, 16, 1)
    part.rows, part.vocab, part.hidden, part.weight, part.targets, part.dloss = len(some), p.vocab, p.hidden[some], p.weight, p.targets[some], p.dloss[some]
    want = part.exact()
    assert ((lse[some].double() - want[4]).abs() <= want[3].amax(1) + 500 * 2.0 ** -24 + 2.0 ** -21 * want[4].abs()).all()
    part_dh, _ = part.check_backward(kt, lse[some])
    # another order of adding the same terms: the difference is within the sums' part of the bound and one step of the result
    assert ((dh[some].float() - part_dh.float()).abs() <= 4 * U16 * part_dh.float().abs() + 4 * U16 * part_dh.float().abs().mean()).all()
    columns = torch.tensor([0, 255, 32767, 32768, 65535, 65536, 65835], device="cuda")
    prob = torch.exp(p.hidden.double() @ p.weight[columns].double().t() - lse.double()[:, None]) * p.dloss.double()[:, None]
    prob -= (p.targets[:, None] == columns[None, :]) * p.dloss.double()[:, None]
    exact, sizes = prob.t() @ p.hidden.double(), prob.abs().t() @ p.hidden.double().abs()
    assert ((dw[columns].double() - exact).abs() <= 2 * U16 * sizes + U16 * exact.abs()).all()


def test_few_rows_share_the_vocabulary(kt):
    """dhidden of few tiles is summed in shares; the last ends inside a stage."""
    p = Problem(130, 136, 40001, 0.1, pad=8)
    p.check_backward(kt, p.check_forward(kt), dlse=p.dlse)


@pytest.mark.parametrize("rows", [3, 400])
def test_targets_past_the_vocabulary(kt, rows):
    p = Problem(rows, 64, 300)
    want, want_lse = p.forward(kt)
    p.targets[1] = 300
    p.targets[2] = 2 ** 40
    loss, lse = p.forward(kt)
    assert torch.isnan(loss[1:3]).all() and torch.equal(loss[3:], want[3:]) and torch.equal(loss[:1], want[:1]) and torch.equal(lse, want_lse)
    dh, dw = p.backward(kt, lse)
    assert torch.isnan(dh[1:3]).all() and not torch.isnan(dh[3:]).any() and torch.isnan(dw).all()


def test_large_logits(kt):
    """Logits of some hundreds: exponentials of most underflow, none overflows."""
    p = Problem(200, 64, 1000, scale=64.0)
    lse = p.check_forward(kt)
    assert lse.abs().max() > 150 and torch.isfinite(lse).all()
    p.check_backward(kt, lse)


def test_non_finite_rows_stay_by_themselves(kt):
    p = Problem(300, 64, 500)
    want, _ = p.forward(kt)
    p.hidden[7] = float("nan")
    loss, lse = p.forward(kt)
    assert torch.isnan(loss[7]) and torch.isnan(lse[7])
    keep = torch.arange(300, device="cuda") != 7
    assert torch.equal(loss[keep], want[keep])


def test_no_rows(kt):
    w = torch.randn(10, 16, device="cuda").to(BF16)
    h, t, f, dw = torch.empty(0, 16, dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), torch.full((10, 16), 3.0, dtype=BF16, device="cuda")
    work = torch.empty(16, dtype=torch.uint8, device="cuda")
    kt.kt_xent_forward(h, w, t, f, f, work)
    kt.kt_xent_backward(f, h, w, t, f, h, dw, work)
    assert (dw == 0).all()


def test_gradient_against_differences(kt):
    """d loss along a direction, by central differences in 64 bits, against the gradients."""
    p = Problem(40, 32, 200, 0.1)
    _, lse = p.forward(kt)
    dh, dw = p.backward(kt, lse, p.dlse)
    gen = torch.Generator().manual_seed(3)
    uh, uw = (torch.randn(n, 32, generator=gen, dtype=torch.float64).cuda() for n in (40, 200))
    used, h, w = p.targets >= 0, p.hidden.double(), p.weight.double()

    def value(step):
        logits = (h + step * uh) @ (w + step * uw).t()
        each = torch.logsumexp(logits, 1)
        loss = each - logits.gather(1, p.targets.clamp(min=0)[:, None])[:, 0]
        return torch.where(used, p.dloss.double() * loss + p.dlse.double() * each, 0.0).sum()

    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    mine = (dh.double() * uh).sum() + (dw.double() * uw).sum()
    sizes = (dh.double() * uh).abs().sum() + (dw.double() * uw).abs().sum()
    assert (slope - mine).abs() <= 2 * U16 * sizes             # two roundings to bf16 on the way to each element


def test_the_same_bits_again_and_captured(kt):
    """Two calls give the same bits; a recorded call reads what its inputs hold when it is replayed."""
    p, q = Problem(700, 136, 3001, 0.1), Problem(700, 136, 3001, 0.4, seed=9)
    first = [*p.forward(kt)]
    first += p.backward(kt, first[1])
    second = [*p.forward(kt)]
    second += p.backward(kt, second[1])
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    loss, lse, dh, dw = (torch.empty_like(t) for t in first)
    work, back = p.work(kt, False), p.work(kt, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kt.kt_xent_forward(p.hidden, p.weight, p.targets, loss, lse, work)
        kt.kt_xent_backward(p.dloss, p.hidden, p.weight, p.targets, lse, dh, dw, back)
    for x in (p, q):
        want = [*x.forward(kt)]
        want += x.backward(kt, want[1])
        for n in ("hidden", "weight", "targets", "dloss"):
            getattr(p, n).copy_(getattr(x, n))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dh, dw)))


def test_two_calls_at_once(kt):
    """On streams of their own, with workspaces of their own."""
    problems, streams, got = [Problem(700, 64, 9000, 0.1, seed=i) for i in range(2)], [torch.cuda.Stream() for _ in range(2)], []
    want = []
    for p in problems:
        loss, lse = p.forward(kt)
        want.append([loss, lse, *p.backward(kt, lse)])
    buffers = [([torch.empty_like(t) for t in w], p.work(kt, False), p.work(kt, True)) for w, p in zip(want, problems)]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, s, (outs, work, back) in zip(problems, streams, buffers):
            kt.kt_xent_forward(p.hidden, p.weight, p.targets, outs[0], outs[1], work, stream=s)
            kt.kt_xent_backward(p.dloss, p.hidden, p.weight, p.targets, outs[1], outs[2], outs[3], back, stream=s)
    torch.cuda.synchronize()
    for w, (outs, _, _) in zip(want, buffers):
        assert all(torch.equal(a, b) for a, b in zip(w, outs))


def test_on_another_stream(kt):
    p = Problem(300, 64, 4000)
    want = p.forward(kt)
    stream, loss, lse, work = torch.cuda.Stream(), *(torch.empty(300, device="cuda") for _ in range(2)), p.work(kt, False)
    stream.wait_stream(torch.cuda.current_stream())
    kt.kt_xent_forward(p.hidden, p.weight, p.targets, loss, lse, work, stream=stream)
    stream.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(lse, want[1])
