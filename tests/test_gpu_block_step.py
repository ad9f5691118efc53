"""A training step through the whole chain: operators on ranks with unequal shares, gradients
synchronised, against a plain fp32 block on the whole batch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def step():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")
    from paper_2505_10183_b200 import block_step
    torch.cuda.set_device(0)
    return block_step


@pytest.mark.parametrize("tokens,width,batch", [(96, 256, 8), (200, 512, 11)])
def test_gradients_of_a_synchronised_step(step, tokens, width, batch):
    """Between the inputs and a gradient lie some 20 roundings to bf16 (at most 2^-8 each, 2^-9.8 rms) and two
    8-bit checkpoints (steps of 1/127 of a block's largest value, some 3.3 times its rms: 0.75 % rms): 1.2 %
    if they were independent and added up, and four times that at the most."""
    shares, errors = step.example(tokens, width, batch)
    assert sum(shares) == batch and shares[0] >= shares[3]
    for name, error in errors.items():
        assert error <= 0.05, (name, errors)


def test_shares_do_not_change_the_gradient(step):
    """The same batch cut in other ways gives the same gradient up to bf16's roundings of the ranks' parts."""
    shape = step.Shape(width=256, heads=4, heads_kv=2, hidden=512)
    params = step.parameters(shape, 3)
    gen = torch.Generator().manual_seed(4)
    x, dz = (torch.randn(8, 64, 256, generator=gen).to(device="cuda", dtype=torch.bfloat16) for _ in range(2))
    one = step.synchronised_step(shape, params, x, dz, [8], [0])
    two = step.synchronised_step(shape, params, x, dz, [3, 2, 1, 2], [0, 0, 1, 1])
    for n in step.NAMES:
        a, b = one[n].float(), two[n].float()
        assert (a - b).norm() <= 0.02 * a.norm(), n            # four parts, a handful of roundings of 2^-8 each
