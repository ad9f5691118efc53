"""The gradient of the cross entropy where P goes over the vocabulary in several pieces (half a GiB of bf16 at a time): every row of
both gradients against the formula in 64 bits, those beside the seams between pieces among them, with rows that do not count, a
gradient of lse, and a last piece of one column.  Tolerances as in test_gpu_xent.py: dhidden is added up over the pieces in fp32, which is
within its sums' (vocab / 16 + 64) roundings."""
import pytest
import torch

from test_gpu_xent import TINY, U16, Problem, kt  # noqa: F401 (kt is a fixture)

pytestmark = pytest.mark.gpu


def pieces_of(rows, vocab):
    """First columns of the pieces: as many as 2^29 bytes of P for whole tiles of 128 rows ask for, of equal length in whole 256 columns."""
    room = 2 ** 29 // (2 * (-(-rows // 128) * 128)) // 256 * 256
    count = -(-vocab // max(room, 256))
    length = -(-(-(-vocab // count)) // 256) * 256
    return list(range(0, vocab, length))


def check(p, lse, dh, dw, dlse, at_once=8192):
    """Both gradients, `at_once` rows of P at a time."""
    used = p.targets >= 0
    h, w = torch.where(used[:, None], p.hidden.double(), 0.0), p.weight.double()
    g = torch.where(used, p.dloss.double(), 0.0)
    z = g if dlse is None else g + torch.where(used, dlse.double(), 0.0)
    want_dw, loose_dw, sizes_dw = (torch.zeros(p.vocab, p.dim, dtype=torch.float64, device="cuda") for _ in range(3))
    for i in range(0, p.rows, at_once):
        s = slice(i, min(i + at_once, p.rows))
        a, at = h[s], torch.arange(s.stop - s.start, device="cuda")
        off = (p.dim / 16 + 16) * 2.0 ** -23 * p.scale * (a.abs() @ w.abs().t())
        prob = torch.exp(p.scale * (a @ w.t()) - lse[s].double()[:, None]) * (p.scale * z[s])[:, None]
        prob = torch.where(used[s, None], prob, 0.0)
        loose = prob.abs() * (off + 2.0 ** -21 + 2.0 ** -22 * lse[s].double().abs()[:, None])
        del off
        prob[at, p.targets[s].clamp(min=0)] -= p.scale * g[s]
        loose += U16 * prob.abs() + TINY * (1 + p.scale * z[s].abs())[:, None]
        want = prob @ w
        slack = loose @ w.abs() + (p.vocab / 16 + 64) * 2.0 ** -23 * (prob.abs() @ w.abs()) + TINY * (p.vocab + 1)
        assert ((dh[s].double() - want).abs() <= slack + U16 * (want.abs() + slack)).all(), i
        assert (dh[s][~used[s]] == 0).all()
        want_dw += prob.t() @ a
        prob.abs_()
        sizes_dw += prob.t() @ a.abs()
        loose_dw += (loose + U16 * prob).t() @ a.abs()
    slack = loose_dw + (p.rows / 16 + 64) * 2.0 ** -23 * sizes_dw + TINY * (p.rows + 1)
    bad = ((dw.double() - want_dw).abs() > slack + U16 * (want_dw.abs() + slack)).any(1)
    assert not bad.any(), bad.nonzero()[:8, 0].tolist()


@pytest.mark.parametrize("rows,dim,vocab,ignored,penalty,starts", [(8192, 16, 65836, 0.0, False, [0, 22016, 44032]), (8192, 200, 65836, 0.1, True, [0, 22016, 44032]),
                                                                  (131072, 72, 24577, 0.1, True, list(range(0, 24577, 2048)))])
def test_every_row(kt, rows, dim, vocab, ignored, penalty, starts):
    assert pieces_of(rows, vocab) == starts
    p = Problem(rows, dim, vocab, ignored, pad=8)
    dlse = p.dlse if penalty else None
    lse = p.forward(kt)[1]
    p.hidden[p.targets < 0] = float("nan")
    dh, dw = p.backward(kt, lse, dlse)
    check(p, lse, dh, dw, dlse)


@pytest.mark.parametrize("hidden", [True, False])
def test_one_gradient_alone(kt, hidden):
    p = Problem(8192, 64, 65836, 0.1)
    lse = p.forward(kt)[1]
    both = p.backward(kt, lse, p.dlse)
    one = p.backward(kt, lse, p.dlse, hidden=hidden, weight=not hidden)
    assert torch.equal(one[0], both[0]) if hidden else torch.equal(one[1], both[1])
