"""Inputs of the embedding whose rows overlap or are one row: they are only read, so any stride will do.  An output's rows may not
overlap, nor may those of a gradient that is added to in place."""
import pytest
import torch

F32, BF16, I64, U8 = torch.float32, torch.bfloat16, torch.int64, torch.uint8


@pytest.fixture(scope="module")
def kt():
    from paper_2505_10183_b200 import binding
    return binding


def rows_of(kind, rows, cols, dtype, gen, device):
    """[rows, cols]: one row for all, or each begins 8 elements behind the one before."""
    flat = torch.randn(cols if kind == "one" else (rows - 1) * 8 + cols, generator=gen).to(device=device, dtype=dtype)
    return flat.as_strided((rows, cols), (0 if kind == "one" else 8, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["one", "overlapping"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens,cols,vocab", [(5, 24, 7), (700, 128, 300), (5000, 512, 149), (1200, 37, 90)])
def test_overlapping_inputs(kt, kind, dtype, tokens, cols, vocab):
    """The same sums as of copies, up to the order that another layout may have: fp32's bound of (n + 3) additions, on either side."""
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    torch.cuda.set_device(0)
    gen = torch.Generator().manual_seed(tokens + cols)
    ids = torch.randint(vocab, (tokens,), generator=gen).cuda()
    weight, dout, base = (rows_of(kind, n, cols, dtype, gen, "cuda") for n in (vocab, tokens, vocab))
    out = torch.empty(tokens, cols, dtype=dtype, device="cuda")
    kt.kt_embed_forward(ids, weight, out)
    assert torch.equal(out, weight[ids])                                        # (scale 1: the elements themselves)
    dw = torch.empty(vocab, cols, dtype=dtype, device="cuda")
    kt.kt_embed_backward(dout, ids, dw, torch.empty(kt.kt_embed_workspace(tokens, cols, vocab), dtype=U8, device="cuda"), scale=0.5, base=base)
    sums, sizes = (torch.zeros(vocab, cols, dtype=torch.float64, device="cuda").index_add_(0, ids, t) for t in (dout.double(), dout.double().abs()))
    count = torch.bincount(ids, minlength=vocab)[:, None]
    want, slack = 0.5 * sums + base.double(), 2.0 ** -24 * ((count + 3) * 0.5 * sizes + base.double().abs())
    half_step = 2.0 ** -24 if dtype == F32 else 2.0 ** -8
    assert ((dw.double() - want).abs() <= half_step * (want.abs() + slack) + slack).all()


def test_what_is_refused_of_them(kt):
    """Without a GPU: an expanded input is passed on to the next check (here a workspace that is too small); outputs are refused as ever."""
    with torch.device("cuda" if torch.cuda.is_available() else "cpu"):
        ids, one, dw, work = torch.zeros(5, dtype=I64), torch.zeros(16), torch.zeros(7, 16), torch.zeros(kt.kt_embed_workspace(5, 16, 7), dtype=U8)
        overlapping = torch.zeros(64).as_strided((7, 16), (4, 1))

    def message(*args, **kw):
        with pytest.raises(kt.KtError) as e:
            kt.kt_embed_backward(*args, stream=0, **kw)
        assert e.value.status == kt.KT_ERR_SHAPE
        return str(e.value)

    assert "workspace" in message(one.expand(5, 16), ids, dw, work[:16])
    assert "workspace" in message(one.expand(5, 16), ids, dw, work[:16], base=one.expand(7, 16))
    assert "dweight" in message(one.expand(5, 16), ids, one.expand(7, 16), work)
    assert "dweight" in message(one.expand(5, 16), ids, overlapping, work, base=overlapping)      # added to in place
    with pytest.raises(kt.KtError) as e:
        kt.kt_embed_forward(ids, one.expand(7, 16), one.expand(5, 16), stream=0)
    assert e.value.status == kt.KT_ERR_SHAPE and "out" in str(e.value)
