"""What the tensor functions make of layouts, on the host: the strides that reach the C boundary are the tensors' own, so that rows
which share memory are refused there before anything is launched."""
import pytest
import torch

from paper_2002_09539_amd import binding as B
from paper_2002_09539_amd import operators as ops

A = 0x7F0000000000      # stand-in for device addresses; never dereferenced
BIG = 1 << 60

# (tensor, rows that share memory)
LOGITS = {
    "one row for all": (torch.zeros(1, 8).expand(4, 8), True),
    "a window that slides": (torch.zeros(11).as_strided((4, 8), (1, 1)), True),
    "rows one element short": (torch.zeros(29).as_strided((4, 8), (7, 1)), True),
    "one logit for all": (torch.zeros(1, 1).expand(4, 1), True),
    "side by side": (torch.zeros(4, 8), False),
    "apart": (torch.zeros(4, 11)[:, 2:10], False),
    "one row": (torch.zeros(8).as_strided((1, 8), (3, 1)), False),
    "no rows": (torch.zeros(0, 8), False),
    "a column": (torch.zeros(4, 8)[:, 3:4], False),
}


@pytest.mark.parametrize("name", LOGITS)
def test_row_strides_of_logits(name):
    t, shared = LOGITS[name]
    _, rows, stride = ops._logit_rows(t, "logits")
    vocab = t.shape[1]
    assert rows == t.shape[0] and stride == (t.stride(0) if rows > 1 else vocab)
    last = (rows - 1) * stride + vocab if rows else 0
    assert shared or t.storage_offset() + last <= t.untyped_storage().nbytes() // 4
    if not shared:
        return
    for call in (lambda: B.ols_token_logprobs(rows, vocab, A, B.OLS_F32, stride, A, A, A, A, A, 0, None, None, None, None, None, 0, A, BIG, None),
                 lambda: B.ols_token_logprobs(rows, vocab, A, B.OLS_F32, vocab, A, A, A, A, A, 0, None, None, A, A, A + 4096, stride, A, BIG, None),
                 lambda: B.ols_token_logprobs_grad(rows, vocab, A, B.OLS_F32, stride, A, A, A, A, A, A + 4096, vocab, None),
                 lambda: B.ols_token_logprobs_grad(rows, vocab, A, B.OLS_F32, vocab, A, A, A, A, A, A + 4096, stride, None)):
        with pytest.raises(B.OlsError, match="elements apart"):
            call()


def test_block_gradients_that_need_each_others_operands():
    """dx over x is written last, gradients over the weights first: both at once would read what is overwritten."""
    f = B.ols_ffn()
    f.groups, f.act, f.dtype, f.weight_dtype, f.grad_dtype = 1, B.OLS_ACT_SILU, B.OLS_F32, B.OLS_F32, B.OLS_F32
    f.rows, f.width, f.hidden, f.out = 40, 16, 32, 16
    shapes = dict(x=(40, 16), w_gate=(16, 32), w_up=(16, 32), w_down=(32, 16), dy=(40, 16), dx=(40, 16), g_gate=(16, 32), g_up=(16, 32), g_down=(32, 16))
    for i, (name, (r, c)) in enumerate(shapes.items()):
        setattr(f, name, B.ols_matrix(A + (i << 20), c, r * c))
    f.saved, f.saved_bytes, f.ws, f.ws_bytes = A, BIG, A, BIG
    need = B.ols_gated_ffn_workspace_bytes(f, 1)
    for on in ("x", "dy"):
        for grad, weight in (("g_gate", "w_gate"), ("g_up", "w_up")):
            g = B.ols_ffn.from_buffer_copy(f)
            g.dx.dev, getattr(g, grad).dev = getattr(g, on).dev, getattr(g, weight).dev
            assert B.ols_gated_ffn_workspace_bytes(g, 1) == need
            with pytest.raises(B.OlsError, match="both at once"):
                B.ols_gated_ffn_grad(g, None)


def test_tensors_that_would_be_scaled_twice():
    """In one launch two workgroups would scale the same elements, in no order."""
    assert ops._distinct([], []) and ops._distinct([A, A + 64, 0], [4, 5, 0]) and ops._distinct([0, A, 0], [0, 3, 0])
    assert ops._distinct([A, A, A + 4], [0, 7, 1])                                  # an empty slice in front of a tensor
    assert not ops._distinct([A, A + 64, A], [4, 4, 4])


def test_saved_states_are_whole():
    """One byte for all, every other byte, another type: fewer bytes lie there than the elements say."""
    whole = torch.zeros(4096, dtype=torch.uint8)
    assert ops._saved(whole) == (whole.data_ptr(), 4096) and ops._saved(whole[:0]) == (None, 0)
    for t in (whole[:1].expand(4096), whole[::2], whole.view(64, 64), whole.float()):
        with pytest.raises(B.OlsError, match="saved"):
            ops._saved(t)


@pytest.mark.parametrize("m", [0, -1])
def test_no_workers(m):
    with pytest.raises(B.OlsError, match="worker"):
        ops._ids(torch.zeros(0, 3, dtype=torch.int32), m)
