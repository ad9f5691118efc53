"""A language model's step without blocks: the embedding, a norm and the loss, of sequences that differ in length."""
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


@pytest.mark.parametrize("tokens,width,vocab,batch", [(96, 256, 1000, 8), (130, 512, 5003, 11)])
def test_no_blocks(step, tokens, width, vocab, batch):
    """The loss is the mean over sequences of the mean over their tokens, with blocks or without.  Between the ids and a
    gradient lie ten roundings to bf16 (2^-9.8 rms each: 0.36 % together) and one 8-bit checkpoint (0.75 % rms): 1.1 % if they added
    up, three times that at the most.  (With a mean over all tokens of a rank, whose sequences differ in
    length, the embedding's gradient is 8 % off, the norm's bias' 8 to 10.)"""
    shares, errors = step.example(tokens, width, 0, vocab, batch)
    assert sum(shares) == batch and set(errors) == {"embed", "norm.weight", "norm.bias"}
    for name, error in errors.items():
        assert error <= 0.033, (name, errors)
