"""Arguments that the embedding, the loss and matrix updates refuse, before anything is launched (no GPU needed: every case is
turned away on the host; where there is a GPU the tensors are there)."""
import ctypes as C

import pytest
import torch

F32, BF16, I64, U8 = torch.float32, torch.bfloat16, torch.int64, torch.uint8


@pytest.fixture(scope="module")
def kt():
    from paper_2505_10183_b200 import binding
    return binding


@pytest.fixture(autouse=True)
def where():
    with torch.device("cuda" if torch.cuda.is_available() else "cpu"):
        yield


def status(kt, call, *args, **kw):
    with pytest.raises(kt.KtError) as e:
        call(*args, stream=0, **kw)
    assert str(e.value)
    return e.value.status


def lookup():
    return torch.zeros(5, dtype=I64), torch.zeros(7, 16), torch.zeros(5, 16)


def test_embedding(kt):
    ids, w, out = lookup()
    f = kt.kt_embed_forward
    assert status(kt, f, ids.int(), w, out) == kt.KT_ERR_SHAPE
    assert status(kt, f, ids[:4], w, out) == kt.KT_ERR_SHAPE
    assert status(kt, f, torch.zeros(10, dtype=I64)[::2], w, out) == kt.KT_ERR_SHAPE
    assert status(kt, f, ids, w[:, :15].contiguous(), out) == kt.KT_ERR_SHAPE
    assert status(kt, f, ids, w.double(), out) == kt.KT_ERR_SHAPE
    assert status(kt, f, ids, torch.zeros(16, 7).t(), out) == kt.KT_ERR_SHAPE
    assert status(kt, f, ids, w, torch.zeros(64).as_strided((5, 16), (8, 1))) == kt.KT_ERR_SHAPE        # rows overlap
    assert status(kt, f, ids, w, out, scale=float("inf")) == kt.KT_ERR_INVALID
    assert status(kt, f, ids, w, out, scale=float("nan")) == kt.KT_ERR_INVALID
    assert status(kt, f, None, w, out) == kt.KT_ERR_INVALID
    assert status(kt, f, ids, w[:0], out) == kt.KT_ERR_SHAPE                                           # no vocabulary


def test_gradient_of_the_embedding(kt):
    ids, dw, dout = lookup()
    work = torch.zeros(kt.kt_embed_workspace(5, 16, 7), dtype=U8)
    b = kt.kt_embed_backward
    assert status(kt, b, dout, ids, dw, None) == kt.KT_ERR_INVALID
    assert status(kt, b, dout, ids, dw, work[:-16]) == kt.KT_ERR_SHAPE
    assert status(kt, b, dout, ids, dw, torch.zeros(1, dtype=U8).expand(work.numel())) == kt.KT_ERR_SHAPE
    assert status(kt, b, dout, ids, dw, torch.zeros(work.numel() + 16, dtype=U8)[8:]) == kt.KT_ERR_ALIGN
    assert status(kt, b, dout, ids[:3], dw, work) == kt.KT_ERR_SHAPE
    assert status(kt, b, dout[:, :8].contiguous(), ids, dw, work) == kt.KT_ERR_SHAPE
    assert status(kt, b, dout, ids, dw, work, base=torch.zeros(7, 16, dtype=BF16)) == kt.KT_ERR_SHAPE
    assert status(kt, b, dout, ids, dw, work, base=torch.zeros(6, 16)) == kt.KT_ERR_SHAPE
    wide = torch.zeros(7 * 32)
    assert status(kt, b, dout, ids, wide.as_strided((7, 16), (32, 1)), work, base=wide.as_strided((7, 16), (16, 1))) == kt.KT_ERR_SHAPE      # itself, otherwise laid out
    assert status(kt, b, dout, ids, torch.zeros(64).as_strided((7, 16), (4, 1)), work) == kt.KT_ERR_SHAPE


def test_workspaces(kt):
    """Enough for the least and the largest, nothing for what would be refused."""
    assert kt.kt_embed_workspace(-1, 8, 8) == kt.kt_embed_workspace(1, 0, 8) == kt.kt_embed_workspace(1, 8, 0) == kt.kt_embed_workspace(1, 8, 2 ** 24 + 1) == 0
    assert kt.kt_embed_workspace(0, 8, 8) > 0
    for back in (False, True):
        assert kt.kt_xent_workspace(0, 8, 8, back) == kt.kt_xent_workspace(2 ** 20 + 1, 8, 8, back) == kt.kt_xent_workspace(1, 8, 2 ** 24 + 1, back) == 0
        assert kt.kt_xent_workspace(1, 8, 1, back) > 0
    # P of a piece is half a GiB at most, whatever the vocabulary
    assert kt.kt_xent_workspace(8192, 64, 2 ** 24, True) < 2 ** 30 < 2 * 8192 * 2 ** 24
    assert kt.kt_orth_workspace(0, 8, 8) == kt.kt_orth_workspace(1, 0, 8) == kt.kt_orth_workspace(1, 8, 2 ** 16 + 1) == 0
    assert kt.kt_orth_workspace(2, 100, 300) >= 2 * 2 * (2 * 100 * 300 + 2 * 100 * 100)


def loss(kt, rows=6, dim=16, vocab=9, backward=False):
    h, w, t, f = torch.zeros(rows, dim, dtype=BF16), torch.zeros(vocab, dim, dtype=BF16), torch.zeros(rows, dtype=I64), torch.zeros(rows)
    work = torch.zeros(kt.kt_xent_workspace(rows, dim, vocab, backward), dtype=U8)
    return [f, h, w, t, f.clone(), h.clone(), w.clone(), work] if backward else [h, w, t, f, f.clone(), work]


def test_loss(kt):
    f = kt.kt_xent_forward

    def refused(which, what, **kw):
        args = loss(kt)
        if which is not None:
            args[which] = what
        return status(kt, f, *args, **kw)

    assert refused(0, torch.zeros(6, 16)) == kt.KT_ERR_SHAPE                    # another type than the weights
    assert refused(0, torch.zeros(6, 24, dtype=BF16)) == kt.KT_ERR_SHAPE
    assert refused(2, torch.zeros(6, dtype=torch.int32)) == kt.KT_ERR_SHAPE
    assert refused(2, torch.zeros(5, dtype=I64)) == kt.KT_ERR_SHAPE
    assert refused(3, torch.zeros(7)) == kt.KT_ERR_SHAPE
    assert refused(4, torch.zeros(6, dtype=BF16)) == kt.KT_ERR_SHAPE
    assert refused(5, None) == kt.KT_ERR_INVALID
    assert refused(5, torch.zeros(64, dtype=U8)) == kt.KT_ERR_SHAPE
    for scale in (0.0, -1.0, float("nan"), 2.0 ** 21, 2.0 ** -21):
        assert refused(None, None, scale=scale) == kt.KT_ERR_INVALID
    assert status(kt, f, *(t.float() if t.dtype == BF16 else t for t in loss(kt))) == kt.KT_ERR_INVALID       # fp32 rows and weights
    odd = loss(kt)
    odd[0], odd[1] = torch.zeros(6, 12, dtype=BF16), torch.zeros(9, 12, dtype=BF16)
    assert status(kt, f, *odd) == kt.KT_ERR_SHAPE                              # dim: a multiple of 8
    assert refused(1, torch.zeros(9 * 20, dtype=BF16).as_strided((9, 16), (20, 1))) == kt.KT_ERR_ALIGN
    assert refused(1, torch.zeros(9 * 16 + 8, dtype=BF16)[4:148].view(9, 16)) == kt.KT_ERR_ALIGN
    assert refused(1, torch.zeros(9 * 16, dtype=BF16).as_strided((9, 16), (8, 1))) == kt.KT_ERR_SHAPE


def test_gradient_of_the_loss(kt):
    b = kt.kt_xent_backward

    def refused(changes, **kw):
        args = loss(kt, backward=True)
        for i, what in changes.items():
            args[i] = what
        return status(kt, b, *args, **kw)

    assert refused({5: None, 6: None}) == kt.KT_ERR_INVALID
    assert refused({5: torch.zeros(6, 16)}) == kt.KT_ERR_SHAPE
    assert refused({6: torch.zeros(9, 16)}) == kt.KT_ERR_SHAPE
    assert refused({6: torch.zeros(9 * 16, dtype=BF16).as_strided((9, 16), (8, 1))}) == kt.KT_ERR_SHAPE
    assert refused({0: torch.zeros(6).expand(6)[:5]}) == kt.KT_ERR_SHAPE
    assert refused({0: torch.zeros(1).expand(6)}) == kt.KT_ERR_SHAPE            # a broadcast gradient needs a copy
    assert refused({}, dlse=torch.zeros(5)) == kt.KT_ERR_SHAPE
    assert refused({7: torch.zeros(1024, dtype=U8)}) == kt.KT_ERR_SHAPE
    assert refused({7: None}) == kt.KT_ERR_INVALID


def test_updates(kt):
    u = kt.kt_orth_update
    x, out = torch.zeros(2, 5, 12), torch.zeros(2, 5, 12, dtype=BF16)
    work = torch.zeros(kt.kt_orth_workspace(2, 5, 12), dtype=U8)
    assert status(kt, u, x, out.float(), work) == kt.KT_ERR_SHAPE
    assert status(kt, u, x, out[:1], work) == kt.KT_ERR_SHAPE
    assert status(kt, u, x[0, 0], out[0, 0], work) == kt.KT_ERR_SHAPE
    assert status(kt, u, x.double(), out, work) == kt.KT_ERR_SHAPE
    assert status(kt, u, x.mT, out.mT, work) == kt.KT_ERR_SHAPE
    assert status(kt, u, x, out, None) == kt.KT_ERR_INVALID
    assert status(kt, u, x, out, work[:-1024]) == kt.KT_ERR_SHAPE
    for steps in (0, -3, 65, 10 ** 12):
        assert status(kt, u, x, out, work, steps=steps) == kt.KT_ERR_INVALID
    assert status(kt, u, x, out, work, scale=float("nan")) == kt.KT_ERR_INVALID
    for coefficients in ((9.0, 0.0, 0.0), (2.5, 0.0, 0.0), (float("nan"), 0.0, 0.0), (3.4445, -4.775, 3.0)):
        assert status(kt, u, x, out, work, coefficients=coefficients) == kt.KT_ERR_INVALID, coefficients
    room = torch.zeros(400, dtype=BF16)
    for strides in ((12, 12, 1), (60, 8, 1), (40, 12, 1), (0, 12, 1)):           # rows or matrices overlap
        assert status(kt, u, x, room.as_strided((2, 5, 12), strides), work) == kt.KT_ERR_SHAPE, strides
    assert status(kt, u, torch.zeros(1).expand(2, 5, 12).contiguous().as_strided((2, 5, 12), (60, 8, 1)), out, work) == kt.KT_ERR_SHAPE


def test_tensors_of_another_place(kt):
    if not torch.cuda.is_available():
        pytest.skip("needs a device that they could be mistaken for")
    ids, w, out = lookup()
    assert status(kt, kt.kt_embed_forward, ids.cpu(), w, out) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_embed_forward, ids, w.cpu(), out) == kt.KT_ERR_INVALID
    args = loss(kt)
    args[2] = args[2].cpu()
    assert status(kt, kt.kt_xent_forward, *args) == kt.KT_ERR_INVALID


def test_c_entries_refuse_bad_addresses_and_sizes(kt):
    lib = kt._lib
    x = torch.zeros(4096)
    p = x.data_ptr() // 16 * 16 + 16
    embed, xent, orth = lib.kt_embed_forward, lib.kt_xent_forward, lib.kt_orth_update
    assert embed(p, p, 16, 0, p, 16, 4, 16, 8, 7, 1.0, None) == kt.KT_ERR_INVALID
    assert embed(p + 4, p, 16, 0, p, 16, 4, 16, 8, 0, 1.0, None) == kt.KT_ERR_ALIGN
    assert embed(p, p + 1, 16, 0, p, 16, 4, 16, 8, 0, 1.0, None) == kt.KT_ERR_ALIGN
    assert embed(None, p, 16, 0, p, 16, 4, 16, 8, 0, 1.0, None) == kt.KT_ERR_INVALID
    assert embed(p, None, 16, 0, p, 16, 4, 16, 8, 0, 1.0, None) == kt.KT_ERR_INVALID
    assert embed(p, p, 16, 0, p, 16, -1, 16, 8, 0, 1.0, None) == kt.KT_ERR_SHAPE
    assert embed(p, p, 16, 0, p, 16, 1 << 31, 16, 8, 0, 1.0, None) == kt.KT_ERR_SHAPE
    assert xent(p, 16, p, 16, p, p, p, p, 1 << 30, 4, 16, 8, 0, 1.0, None) == kt.KT_ERR_INVALID                # fp32
    assert xent(p + 8, 16, p, 16, p, p, p, p, 1 << 30, 4, 16, 8, 1, 1.0, None) == kt.KT_ERR_ALIGN
    assert xent(p, 16, p, 16, p + 4, p, p, p, 1 << 30, 4, 16, 8, 1, 1.0, None) == kt.KT_ERR_ALIGN
    assert xent(p, 16, p, 16, p, p + 2, p, p, 1 << 30, 4, 16, 8, 1, 1.0, None) == kt.KT_ERR_ALIGN
    assert xent(p, 16, p, 16, p, p, None, p, 1 << 30, 4, 16, 8, 1, 1.0, None) == kt.KT_ERR_INVALID
    assert xent(p, 16, p, 16, p, p, p, p, 1 << 40, (1 << 20) + 1, 16, 8, 1, 1.0, None) == kt.KT_ERR_SHAPE
    assert xent(p, 16, p, 16, p, p, p, p, 1 << 30, 4, 16, 0, 1, 1.0, None) == kt.KT_ERR_SHAPE
    s, c = (C.c_int64 * 2)(64, 8), (C.c_float * 3)(3.4445, -4.775, 2.0315)
    assert orth(p, s, 3, p, s, p, 1 << 30, 1, 8, 8, 5, c, 1.0, None) == kt.KT_ERR_INVALID
    assert orth(p + 2, s, 0, p, s, p, 1 << 30, 1, 8, 8, 5, c, 1.0, None) == kt.KT_ERR_ALIGN
    assert orth(p, s, 0, p + 1, s, p, 1 << 30, 1, 8, 8, 5, c, 1.0, None) == kt.KT_ERR_ALIGN
    assert orth(p, None, 0, p, s, p, 1 << 30, 1, 8, 8, 5, c, 1.0, None) == kt.KT_ERR_INVALID
    assert orth(p, s, 0, p, s, p, 1 << 30, 1, 8, 8, 5, None, 1.0, None) == kt.KT_ERR_INVALID
    assert orth(p, s, 0, p, s, p + 8, 1 << 30, 1, 8, 8, 5, c, 1.0, None) == kt.KT_ERR_ALIGN
    assert orth(p, s, 0, p, s, p, 1 << 30, 1, 1 << 17, 8, 5, c, 1.0, None) == kt.KT_ERR_SHAPE
    assert lib.kt_last_error(None)
