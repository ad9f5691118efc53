"""Updates orthogonalised by Newton-Schulz products against the formula in 64 bits, on the GPU.

Tolerance, in the 2-norm relative to the result: a step rounds X, A and the factor to fp16, at most 2^-11 relative to each
element and some half of that on average.  Relative to the next X, at singular values near one, the rounding of X
counts once, of the factor once, of A |b| + 2 |c| = 9 times over 0.7 (the smallest value that a step takes one to): 15
roundings' worth, independent from step to step: 15 * 2^-12 * sqrt(5) = 0.8 % after five; 0.2 % more for the result in bf16."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOLERANCE = 0.01
MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def kt():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import binding
    torch.cuda.set_device(0)
    return binding


def exact(x, steps=5, coefficients=MUON, scale=1.0):
    a, b, c = (float(torch.tensor(v, dtype=F32)) for v in coefficients)
    y = x.double()
    y = y / torch.linalg.matrix_norm(y, keepdim=True)
    tall = y.size(-2) > y.size(-1)
    y = y.mT if tall else y
    for _ in range(steps):
        gram = y @ y.mT
        y = a * y + (b * gram + c * gram @ gram) @ y
    return scale * (y.mT if tall else y)


def update(kt, x, out=None, **kw):
    out = torch.full(x.shape, float("nan"), dtype=BF16, device="cuda") if out is None else out
    batch = x.size(0) if x.dim() == 3 else 1
    work = torch.full((kt.kt_orth_workspace(batch, x.size(-2), x.size(-1)),), 255, dtype=torch.uint8, device="cuda")
    kt.kt_orth_update(x, out, work, **kw)
    return out


def far(got, want):
    return float((got.double() - want).norm() / want.norm())


def normal(*shape, seed=0, dtype=F32):
    gen = torch.Generator().manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("shape", [(1, 1), (1, 50), (50, 1), (2, 3), (16, 16), (63, 65), (64, 200), (200, 64), (127, 129), (128, 128), (129, 130), (256, 384), (384, 250), (500, 333), (333, 1030), (1111, 97),
                                   (3, 40, 70), (5, 130, 129), (2, 257, 64), (7, 64, 257)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_cta_to_a_tile(kt, shape, dtype):
    x = normal(*shape, dtype=dtype)
    assert far(update(kt, x, scale=0.7), exact(x, scale=0.7)) <= TOLERANCE


@pytest.mark.parametrize("shape", [(3000, 2900), (2900, 3010), (8, 1024, 1000), (9, 1100, 1030), (75, 200, 136), (75, 130, 300)])
def test_pairs_of_ctas(kt, shape):
    x = normal(*shape, dtype=BF16)
    assert far(update(kt, x), exact(x)) <= TOLERANCE


def test_each_matrix_on_its_own(kt):
    """In a batch, on its own, scaled: the same bits; zeros stay zeros, and what is not finite stays where it is."""
    x = normal(6, 70, 100)
    got = update(kt, x)
    assert torch.equal(update(kt, x[2]), got[2])
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** -90
    x[3] = 0.0
    x[4, 3, 5] = float("inf")
    x[5, 0, 0] = float("nan")
    again = update(kt, x)
    assert torch.equal(again[:3], got[:3])
    assert (again[3] == 0).all() and torch.isnan(again[4:]).all()


@pytest.mark.parametrize("shape", [(1, 50), (716, 2), (4, 465), (465, 4), (13, 65), (64, 640), (64, 700), (77, 835), (8000, 120), (200, 300), (384, 256), (200, 700), (300, 3000), (2500, 260)])
def test_few_singular_values_and_alike(kt, shape):
    """Nothing averages out where there are few, or all are moved the same way.  A's diagonal, whose rounding would move them all, is not
    rounded to fp16, which leaves of the header's 15 roundings X's one, the factor's one and A's beside its diagonal, half of its norm at
    most: (1 + 1 + 13 / 2) 2^-12 / sqrt(3) each on average, and independent in five steps: 0.27 %; with the result's own, 2^-9 / sqrt(3) = 0.11 to 0.19 %: 0.33 %."""
    for seed in range(3):
        x = normal(*shape, seed=seed)
        assert far(update(kt, x), exact(x)) <= 0.0033


@pytest.mark.parametrize("shape", [(128, 640), (640, 128), (128, 641), (641, 128), (129, 640), (640, 129), (64, 640), (65, 577), (1, 640), (640, 1), (3, 128, 576), (3, 513, 120), (200, 100, 330)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_matrix_to_a_cta(kt, shape, dtype):
    """Up to 128 x 640, and a little more."""
    x = normal(*shape, dtype=dtype)
    assert far(update(kt, x, scale=0.7), exact(x, scale=0.7)) <= TOLERANCE


@pytest.mark.parametrize("shape", [(100, 70), (120, 600), (140, 200), (200, 140), (300, 500)])
def test_any_magnitude(kt, shape):
    """Powers of two change nothing, down to fp32's smallest numbers; zeros stay zeros, and what is not finite stays in its matrix."""
    x = normal(6, *shape)
    x = x.sign() * x.abs().clamp(2.0 ** -9, 8.0).bfloat16().float()       # 17 powers of two and 8 bits: exact wherever they are scaled to here
    got = update(kt, x)
    x[0] *= 2.0 ** 120
    x[1] *= 2.0 ** -126
    x[3] = 0.0
    x[4, 3, 5] = float("inf")
    x[5, 0, 0] = float("nan")
    again = update(kt, x)
    assert torch.equal(again[:3], got[:3])
    assert (again[3] == 0).all() and torch.isnan(again[4:]).all()


@pytest.mark.parametrize("shape", [(90, 60), (61, 300), (150, 200), (210, 140)])
def test_room_around_the_output(kt, shape):
    rows, cols = shape
    x = normal(4, *shape)
    want = update(kt, x)
    for left, right in ((0, 0), (1, 8), (8, 1), (0, -cols % 8)):
        out = torch.full((4, rows + 1, left + cols + right), 5.0, dtype=BF16, device="cuda")
        inner = out[:, :rows, left:left + cols]
        update(kt, x, inner)
        assert torch.equal(inner, want)
        inner.fill_(5.0)
        assert (out == 5).all()


def test_strides(kt):
    x = normal(4, 60, 90)
    want = update(kt, x)
    wide = torch.full((4, 60, 101), float("nan"), device="cuda")
    wide[:, :, 3:93] = x
    out = torch.full((4, 60, 99), 5.0, dtype=BF16, device="cuda")
    update(kt, wide[:, :, 3:93], out[:, :, 1:91])
    assert torch.equal(out[:, :, 1:91], want) and (out[:, :, 0] == 5).all() and (out[:, :, 91:] == 5).all()
    room = torch.full((4, 60, 96), 5.0, dtype=BF16, device="cuda")                       # rows at multiples of 16 bytes, which end inside one
    update(kt, x[:, :, :83].contiguous(), room[:, :, :83])
    assert far(room[:, :, :83], exact(x[:, :, :83])) <= TOLERANCE and (room[:, :, 83:] == 5).all()
    turned = torch.empty(60, 4, 90, dtype=BF16, device="cuda").transpose(0, 1)           # rows of all matrices in turn
    update(kt, x.transpose(0, 1).contiguous().transpose(0, 1), turned)
    assert torch.equal(turned, want)


def test_a_broadcast_batch(kt):
    x = normal(70, 100)
    got = update(kt, x.expand(3, 70, 100))
    assert torch.equal(got[0], update(kt, x)) and torch.equal(got[1], got[0]) and torch.equal(got[2], got[0])


def test_a_matrix_of_low_rank(kt):
    """In the directions that x does not have, a rounding of X is raised by a = 3.4445 in every step that follows, where the
    header's tolerance is for directions that x has.  X_0 has the norm 1 and the later ones at most 1.2 sqrt(2) = 1.7, of which
    2^-12 is rounded on average: 2^-12 (a^5 + 1.7 (a^4 + a^3 + a^2 + a)) = 0.2, relative to a result of at least
    0.68 sqrt(2) = 0.96."""
    x = normal(300, 2) @ normal(2, 200, seed=1)
    got, want = update(kt, x), exact(x)
    assert far(got, want) <= 0.21
    # and in the directions that it has, as ever
    u, _, v = torch.linalg.svd(x.double(), full_matrices=False)
    inside = u[:, :2].mT @ got.double() @ v[:2].mT
    assert far(inside, u[:, :2].mT @ want @ v[:2].mT) <= TOLERANCE


def test_what_it_is_for(kt):
    """Singular values end up between 0.65 and 1.25 (where the polynomial of five steps takes all that are not tiny)."""
    x = normal(200, 600)
    s = torch.linalg.svdvals(update(kt, x).double())
    assert 0.65 <= float(s.min()) and float(s.max()) <= 1.25


@pytest.mark.parametrize("steps,coefficients", [(1, MUON), (3, MUON), (10, (1.5, -0.5, 0.0)), (12, (1.875, -1.25, 0.375))])
def test_other_polynomials(kt, steps, coefficients):
    x = normal(130, 260)
    assert far(update(kt, x, steps=steps, coefficients=coefficients), exact(x, steps, coefficients)) <= TOLERANCE


def test_captured(kt):
    x, out = normal(2, 150, 100), torch.empty(2, 150, 100, dtype=BF16, device="cuda")
    work = torch.empty(kt.kt_orth_workspace(2, 150, 100), dtype=torch.uint8, device="cuda")
    kt.kt_orth_update(x, out, work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kt.kt_orth_update(x, out, work)
    for seed in (4, 5):
        x.copy_(normal(2, 150, 100, seed=seed))
        graph.replay()
        assert torch.equal(out, update(kt, x))
