"""Arguments that the training operators refuse, before anything is launched (no GPU needed: every
case is turned away on the host; where there is a GPU the tensors are there)."""
import pytest
import torch

F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8


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


def test_sizes_of_a_checkpoint(kt):
    for cols in (1, 15, 16, 17, 127, 128, 129, 1000):
        assert kt.kt_ckpt_pitch(cols) == -(-cols // 16) * 16 and kt.kt_ckpt_blocks(cols) == -(-cols // 128)
    assert kt.kt_norm_workspace(0, 64) == 0 and kt.kt_norm_workspace(1, 64) == 2 * 64 * 4
    assert kt.kt_norm_workspace(10 ** 6, 64) == kt.kt_norm_workspace(10 ** 7, 64)      # bounded in the rows


def test_refused_matrices(kt):
    x, c, s = torch.zeros(4, 32), torch.zeros(4, 32, dtype=I8), torch.zeros(4, 1)
    w = torch.zeros(32)
    assert status(kt, kt.kt_norm_forward, x.double(), w, w, x.double()) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w, w, torch.zeros(4, 33)) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w, w, x.to(BF16)) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x.t(), w, w, x.t()) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w, w.to(BF16), x) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w[:31], None, x) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w, w, x, torch.zeros(5)) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_norm_forward, x, w, w, x, codes=c) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_norm_forward, x, w, w, x, eps=float("nan")) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_norm_forward, x, w, w, x, eps=-1.0) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_ckpt_store, x, c[:, :16], s) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_ckpt_store, x, c, torch.zeros(4, 2)) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_ckpt_restore, None, None, x) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_act_forward, x, x, kind="tanh") == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_act_forward, x, x, kind=7) == kt.KT_ERR_INVALID
    overlapping = torch.zeros(64).as_strided((4, 32), (8, 1))
    assert status(kt, kt.kt_act_forward, x, overlapping) == kt.KT_ERR_SHAPE


def test_refused_backward_sources(kt):
    x, c, s, r = torch.zeros(4, 32), torch.zeros(4, 32, dtype=I8), torch.zeros(4, 1), torch.zeros(4)
    w, ws = torch.zeros(32), torch.zeros(kt.kt_norm_workspace(4, 32), dtype=torch.uint8)
    back = kt.kt_norm_backward
    assert status(kt, back, x, w, r, x, w, w, ws) == kt.KT_ERR_INVALID                              # neither source
    assert status(kt, back, x, w, r, x, w, w, ws, x=x, mean=r, codes=c, scales=s) == kt.KT_ERR_INVALID   # both
    assert status(kt, back, x, w, r, x, w, w, ws, x=x) == kt.KT_ERR_INVALID                         # no mean
    assert status(kt, back, x, w, None, x, w, w, ws, codes=c, scales=s) == kt.KT_ERR_INVALID        # no rstd
    assert status(kt, back, x, w, r, x, w, w, None, codes=c, scales=s) == kt.KT_ERR_INVALID
    assert status(kt, back, x, w, r, x, w, w, ws[:-16], codes=c, scales=s) == kt.KT_ERR_SHAPE
    assert status(kt, back, x, w, r, x, w, w.to(BF16), ws, codes=c, scales=s) == kt.KT_ERR_SHAPE
    assert status(kt, kt.kt_act_backward, x, None, None, x) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_act_backward, x, c, s, x, x=x) == kt.KT_ERR_INVALID


def test_tensors_in_host_memory_are_refused_where_there_is_a_device(kt):
    if not torch.cuda.is_available():
        pytest.skip("needs a device that they could be mistaken for")
    x, host = torch.zeros(4, 32), torch.zeros(4, 32, device="cpu")
    assert status(kt, kt.kt_act_forward, host, host) == kt.KT_ERR_INVALID
    assert status(kt, kt.kt_act_forward, x, host) == kt.KT_ERR_INVALID
    with pytest.raises(kt.KtError):
        kt.kt_act_forward([1.0], x, stream=0)


def test_c_entries_refuse_bad_addresses_and_types(kt):
    lib = kt._lib
    x = torch.zeros(4, 32)
    p = x.data_ptr()
    c = torch.zeros(256, dtype=I8).data_ptr() // 16 * 16 + 16
    assert lib.kt_act_forward(p, 32, None, 32, None, None, 4, 32, 0, 0, None) == kt.KT_ERR_INVALID
    assert lib.kt_act_forward(p + 2, 32, p, 32, None, None, 4, 32, 0, 0, None) == kt.KT_ERR_ALIGN
    assert lib.kt_act_forward(p, 32, p, 32, c + 8, p, 4, 32, 0, 0, None) == kt.KT_ERR_ALIGN
    assert lib.kt_act_forward(p, 32, p, 32, None, None, 4, 32, 5, 0, None) == kt.KT_ERR_INVALID
    assert lib.kt_act_forward(p, 32, p, 32, None, None, -1, 32, 0, 0, None) == kt.KT_ERR_SHAPE
    assert lib.kt_act_forward(p, 32, p, 32, None, None, 4, 0, 0, 0, None) == kt.KT_ERR_SHAPE
    assert lib.kt_act_forward(p, 32, p, 32, None, None, 1 << 60, 32, 0, 0, None) == kt.KT_ERR_SHAPE
    assert lib.kt_ckpt_store(p, 31, c, p, 4, 32, 0, None) == kt.KT_ERR_SHAPE
    assert lib.kt_norm_forward(p, 32, p, p, 9, p, 32, None, None, None, None, 4, 32, 0, 1e-5, None) == kt.KT_ERR_INVALID
    assert lib.kt_last_error(None)


def heads(*shape):
    return torch.zeros(*shape, dtype=BF16)


def attention(kt, len_q=16, len_kv=16, dim=64):
    """Arguments of kt_attn_backward in their order, for 2 sequences, 4 heads on 2; those of the forward pass are 1 ... 5 of them."""
    q, k = heads(2, len_q, 4, dim), heads(2, len_kv, 2, dim)
    work = torch.zeros(max(1, kt.kt_attn_workspace(q, k)), dtype=torch.uint8)
    return [heads(2, len_q, 4, dim), q, k, heads(2, len_kv, 2, dim), heads(2, len_q, 4, dim), torch.zeros(2, 4, len_q), heads(2, len_q, 4, dim),
            heads(2, len_kv, 2, dim), heads(2, len_kv, 2, dim), work]


def test_workspaces_that_are_smaller_than_they_look(kt):
    """An expanded tensor counts bytes that it does not have, a strided one bytes between those of others."""
    x, c, s, r, w = torch.zeros(4, 32), torch.zeros(4, 32, dtype=I8), torch.zeros(4, 1), torch.zeros(4), torch.zeros(32)
    need = kt.kt_norm_workspace(4, 32)
    for work in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2]):
        assert status(kt, kt.kt_norm_backward, x, w, r, x, w, w, work, codes=c, scales=s) == kt.KT_ERR_SHAPE
    args = attention(kt)
    need = args[9].numel()
    for work in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2]):
        assert status(kt, kt.kt_attn_backward, *args[:9], work) == kt.KT_ERR_SHAPE


def test_c_entries_refuse_row_statistics_at_odd_addresses(kt):
    lib = kt._lib
    x, w, ws = torch.zeros(4, 32), torch.zeros(32), torch.zeros(kt.kt_norm_workspace(4, 32) + 16, dtype=torch.uint8)
    p, r, at = x.data_ptr(), torch.zeros(8).data_ptr(), ws.data_ptr() // 16 * 16 + 16

    def forward(mean, rstd):
        return lib.kt_norm_forward(p, 32, w.data_ptr(), None, 0, p, 32, mean, rstd, None, None, 4, 32, 0, 1e-5, None)

    def backward(mean, rstd):
        return lib.kt_norm_backward(p, 32, p, 32, mean, None, None, rstd, None, 0, p, 32, None, None, at, ws.numel() - 16, 4, 32, 0, None)

    for call in (forward, backward):
        assert call(r + 1, r) == kt.KT_ERR_ALIGN
        assert call(r, r + 2) == kt.KT_ERR_ALIGN


@pytest.mark.parametrize("which,name", [(3, "out"), (6, "dq"), (7, "dk"), (8, "dv")])
def test_attention_outputs_that_overlap_themselves(kt, which, name):
    """Tokens, heads or sequences that share elements would be written by several CTAs at once; inputs may do so."""
    for len_q, len_kv in ((16, 16), (0, 16), (16, 0)):
        args = attention(kt, len_q, len_kv)
        if name == "out":                                              # of the forward pass
            args = [args[1], args[2], args[3], args[6], args[5]]
            call = kt.kt_attn_forward
        else:
            call = kt.kt_attn_backward
        B, L, H, D = args[which].shape
        if L == 0:
            continue
        room = torch.zeros(4 * B * L * H * D, dtype=BF16)
        for strides in ((L * H * D, H * D, 8, 1),                      # heads
                        (L * H * D, 8, L * D, 1),                      # tokens
                        (L * H * D, D, D, 1),                          # a token's second head is the next token's first
                        (H * D, H * D, D, 1),                          # sequences
                        (L * H * D, (H - 1) * D + 8, D, 1),            # a token begins inside the last one
                        (L * H * D - 8, H * D, D, 1)):
            args[which] = room.as_strided((B, L, H, D), strides)
            assert status(kt, call, *args) == kt.KT_ERR_SHAPE, strides


def test_attention_outputs_in_any_order_of_dimensions(kt):
    """Layouts without overlaps get past the checks: without a device the call then ends for want of one."""
    if torch.cuda.is_available():
        pytest.skip("runs as a whole there (test_layouts)")
    B, L, H, D = 2, 16, 4, 64
    for strides in ((L * H * D, H * D, D, 1), (L * H * D, D, L * D, 1), (D, B * D, L * B * D, 1), (L * H * 72 + 8, H * 72, 72, 1)):
        args = attention(kt)
        args[6] = torch.zeros(2 * B * L * H * 72, dtype=BF16).as_strided((B, L, H, D), strides)
        assert status(kt, kt.kt_attn_backward, *args) == kt.KT_ERR_CUDA, strides
    args = attention(kt)
    args[2] = torch.zeros(2 * 16 * 2 * 64, dtype=BF16).as_strided((2, 16, 2, 64), (16 * 64, 64, 8, 1))       # an input
    assert status(kt, kt.kt_attn_backward, *args) == kt.KT_ERR_CUDA


def test_limits_of_a_wait(kt):
    for limit in (-1, 60 * 10 ** 9 + 1):
        with pytest.raises(kt.KtError) as e:
            kt.kt_attn_wait_limit(limit)
        assert e.value.status == kt.KT_ERR_INVALID
    kt.kt_attn_wait_limit(2 * 10 ** 9)              # what it is at first
