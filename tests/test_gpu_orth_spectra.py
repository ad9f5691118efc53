"""Orthogonalised updates of matrices as training has them: singular values that fall, or few beside none, where what a rounding to
fp16 leaves in the small directions is raised by up to a = 3.4445 in every step that follows.

Tolerance, in the 2-norm relative to the result.  An element is rounded to fp16 by at most 2^-11 of itself, evenly spread, so by U = 2^-11 / sqrt(3)
rms at the most, and the roundings of a matrix are white: of X (U |X|), of A beside its diagonal (U |R|, which reaches the next X as
(b + c (A_i + A_j)) s_j), and of the factor (U |F| |X| / sqrt(m)).  What becomes of white noise on X in the steps that follow is, to first order,
the derivative of X -> u phi(s) v^T, where phi is the polynomial taken so many times: the symmetric part of the element between
directions i and j goes by (phi(s_i) - phi(s_j)) / (s_i - s_j), the antisymmetric part by (phi(s_i) + phi(s_j)) / (s_i + s_j), and what
lies outside of v by phi(s_i) / s_i.  The squares of all five steps' add up, with the result's own rounding to bf16 (2^-8 / sqrt(3))."""
import math

import pytest
import torch

from test_gpu_orth import BF16, F32, MUON, exact, far, kt, normal, update  # noqa: F401 (kt is a fixture)

U, STEPS = 2.0 ** -11 / math.sqrt(3.0), 5
A, B, C = (float(torch.tensor(v, dtype=F32)) for v in MUON)


def phi(s):
    return s * (A + s * s * (B + s * s * C))


def gain(s, steps, others):
    """Mean square factor by which white noise on a matrix of singular values s and `others` columns more grows in `steps` steps."""
    m, to, slope = len(s), s, torch.ones_like(s)
    for _ in range(steps):
        slope, to = slope * (A + to * to * (3 * B + to * to * 5 * C)), phi(to)
    away, sums = s[:, None] - s, s[:, None] + s
    same, none = away.abs() <= 1e-9 * sums, sums < 1e-30
    minus = torch.where(same, slope[:, None], (to[:, None] - to) / torch.where(same, 1.0, away))
    plus = torch.where(none, A ** steps, (to[:, None] + to) / torch.where(none, 1.0, sums))
    outside = torch.where(s < 1e-30, A ** steps, to / s.clamp(min=1e-30))
    return float(((minus ** 2 + plus ** 2) / 2).sum() + others * (outside ** 2).sum()) / (m * (m + others))


def tolerance(s, others):
    s, m, off, first = s / s.norm(), len(s), 0.0, s
    for step in range(STEPS):
        size, gram, left = float((s * s).sum()), s * s, STEPS - 1 - step
        factor = A + gram * (B + gram * C)
        beside = max(0.0, float((gram * gram).sum()) - float(gram.sum()) ** 2 / m)
        through = float(((B + C * (gram[:, None] + gram)) ** 2 * gram).sum()) / (m * m)
        off += size * gain(s, left + 1, others) + (beside * through + float((factor * factor).sum()) * size / m) * gain(phi(s), left, others)
        s = phi(s)
    return math.sqrt(U * U * off / float((s * s).sum()) + (2.0 ** -8 / math.sqrt(3.0)) ** 2) + of_one_value(first, others)


def of_one_value(s, others):
    """What the factor's diagonal, one value throughout and rounded, adds."""
    if len(s) <= 64 or len(s) + others >= 8 * len(s) or float(s.max() - s.min()) > 1e-9 * float(s.max()):
        return 0.0
    v, off = float(s[0] / s.norm()), 0.0
    for _ in range(STEPS):
        factor = A + v * v * (B + v * v * C)
        off = off * abs(1 + v * v * (2 * B + 4 * C * v * v) / factor) + 2.0 ** -11
        v *= factor
    return off


def spectrum(kind, m):
    i = torch.arange(m, dtype=torch.float64)
    if kind.startswith("to"):
        return 10.0 ** (-float(kind[2:]) * i / max(1, m - 1))
    if kind.endswith("alike"):
        return (i < int(kind.split()[0])).double()
    return 1.0 / (i + 1)


def matrix(shape, kind):
    """[batch,] rows x cols with the singular values of `kind` (each matrix with directions of its own)."""
    rows, cols = shape[-2:]
    m = min(rows, cols)
    s = spectrum(kind, m)
    u, v = (torch.linalg.qr(normal(*shape[:-2], n, m, seed=seed).double())[0] for n, seed in ((rows, 1), (cols, 2)))
    return ((u * s.cuda()) @ v.mT).float(), tolerance(s, max(rows, cols) - m)


KINDS = ["to1", "to3", "to4", "to6", "harmonic", "1 alike", "8 alike", "64 alike", "1000 alike"]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(64, 64), (40, 600), (128, 128), (256, 256), (300, 200), (424, 424), (512, 512), (200, 700), (1000, 300), (16, 512, 512), (50, 40, 700), (17, 800, 700)])
def test_spectra(kt, shape, kind):
    x, most = matrix(shape, kind)
    assert far(update(kt, x, scale=0.7), exact(x, scale=0.7)) <= most


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(128, 128), (256, 256), (512, 512)])
def test_a_gradient_of_few_tokens(kt, shape):
    """A momentum of a rank as low as its tokens are few, in bf16 (whose roundings, not being the kernel's, are x's own): the formula of
    what is given."""
    x = (normal(shape[0], 24, seed=3) @ normal(24, shape[1], seed=4)).to(BF16)
    s = torch.linalg.svdvals(x.double())
    assert far(update(kt, x), exact(x)) <= tolerance(s.cpu(), abs(shape[0] - shape[1]))


def emulated(x):
    """The kernels' roundings in 64 bits: X in fp16 times 2^7, A beside its diagonal 2^14, the factor 2^13."""
    def half(t, unit):
        return (t * unit).to(torch.float16).double() / unit

    y = half(x / x.norm(), 2.0 ** 7)
    for step in range(STEPS):
        gram = y @ y.mT
        beside = half(gram - torch.diag(gram.diagonal()), 2.0 ** 14)
        rounded = beside + torch.diag(gram.diagonal())
        factor = A * torch.eye(len(y), dtype=torch.float64) + B * rounded + C * rounded @ rounded
        y = half(factor, 2.0 ** 13) @ y
        if step + 1 < STEPS:
            y = half(y, 2.0 ** 7)
    return y.to(BF16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(48, 48), (64, 200)])
def test_the_tolerance(rows, cols, kind):
    """The roundings that it counts stay within it, and it is at most four times what they are."""
    gen = torch.Generator().manual_seed(rows + cols)
    u, v = (torch.linalg.qr(torch.randn(n, rows, generator=gen, dtype=torch.float64))[0] for n in (rows, cols))
    s = spectrum(kind, rows)
    x, most = (u * s) @ v.mT, tolerance(s, cols - rows)
    y = x / x.norm()
    for _ in range(STEPS):
        gram = y @ y.mT
        y = A * y + (B * gram + C * gram @ gram) @ y
    off = float((emulated(x).double() - y).norm() / y.norm())
    assert most / 4 <= off <= most
