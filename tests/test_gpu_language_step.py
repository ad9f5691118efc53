"""A language model's training step through the whole chain: embedding, blocks, loss, gradients synchronised over ranks with
unequal shares, orthogonalised update; against a plain fp32 model on the whole batch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def step():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import language_step
    torch.cuda.set_device(0)
    return language_step


@pytest.mark.parametrize("tokens,width,layers,vocab,batch", [(96, 256, 1, 1000, 8), (130, 512, 2, 5003, 11)])
def test_gradients_of_a_synchronised_step(step, tokens, width, layers, vocab, batch):
    """Between the ids and a gradient lie some 20 roundings to bf16 for each block and 10 more for the ends (at most 2^-8 each,
    2^-9.8 rms), and two 8-bit checkpoints to a block and one of the last norm (steps of 1/127 of a block's largest value, some 3.3
    times its rms: 0.75 % rms): 1.9 % for two blocks if they were independent and added up, and four times that at
    the most."""
    shares, errors = step.example(tokens, width, layers, vocab, batch)
    assert sum(shares) == batch and shares[0] >= shares[3] and set(errors) == set(step.names(layers))
    for name, error in errors.items():
        assert error <= 0.08, (name, errors)


def test_update(step):
    """Every matrix moves along a direction whose singular values are near one times the factor of its shape; the others along the gradient."""
    shape = step.Shape(width=128, heads=2, heads_kv=1, hidden=512)
    params = step.parameters(shape, 2, 300, 1)
    gen = torch.Generator().manual_seed(2)
    grads = {n: (torch.randn(p.shape, generator=gen) * 1e-3).to(p) for n, p in params.items()}
    before = {n: p.clone() for n, p in params.items()}
    update = step.Update(2, params, rate=0.5, rate_others=8.0)
    update.step(grads)
    for n, p in params.items():
        moved = (before[n].float() - p.float())
        rounding = 2.0 ** -8 * (before[n].float().abs() + moved.abs())
        if n.partition(".")[2] in step.MATRICES:
            s = torch.linalg.svdvals(moved / 0.5) / max(1.0, p.size(0) / p.size(1)) ** 0.5
            # the smallest of random matrices of these shapes are not tiny; what the rounding of p adds is at most its norm
            assert float(s.max()) <= 1.25 + 2 * float(rounding.norm()) and float(s.mean()) >= 0.65
        else:
            assert ((moved - 8.0 * grads[n].float()).abs() <= rounding + 2.0 ** -8 * 8.0 * grads[n].float().abs()).all()


def test_one_rank_or_four(step):
    """The same batch cut in other ways gives the same losses, and the same gradient up to bf16's roundings of the ranks' parts."""
    shape = step.Shape(width=256, heads=4, heads_kv=2, hidden=512)
    params, data = step.parameters(shape, 1, 700, 3), step.batch_of(700, 8, 64, 4)
    loss, one = step.synchronised_step(shape, 1, params, data, [8], [0])
    parts, two = step.synchronised_step(shape, 1, params, data, [3, 2, 1, 2], [0, 0, 1, 1])
    # the stock matrix products between may round otherwise for other numbers of rows: some ten steps of bf16, rms, of rows of norm one
    assert ((loss - parts).abs() <= 0.05).all() and (loss[data[1] < 0] == 0).all()
    for n in one:
        a, b = one[n].float(), two[n].float()
        assert (a - b).norm() <= 0.02 * a.norm(), n            # four parts, a handful of roundings of 2^-8 each
