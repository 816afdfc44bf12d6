"""Layouts that the tensor functions refuse, and layouts that they have to take."""
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_and_gradients_whose_rows_share_memory_are_refused(dtype):
    ops = _ops()
    whole = torch.zeros(4, 9, dtype=dtype, device="cuda")
    t, g = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    r = ops.token_logprobs(whole, t)
    flat = torch.zeros(36, dtype=dtype, device="cuda")
    for shared in (flat[:9].expand(4, 9), flat.as_strided((4, 9), (1, 1)), flat.as_strided((4, 9), (8, 1))):
        for call in (lambda: ops.token_logprobs(shared, t), lambda: ops.token_logprobs_with_grad(shared, t, g),
                     lambda: ops.token_logprobs_with_grad(whole, t, g, out=shared), lambda: ops.token_logprobs_grad(shared, t, r, g),
                     lambda: ops.token_logprobs_grad(whole, t, r, g, out=shared)):
            with pytest.raises(B.OlsError):
                call()
    column = torch.zeros(1, 1, dtype=dtype, device="cuda").expand(4, 1)
    with pytest.raises(B.OlsError):
        ops.token_logprobs(column, t)
    assert ops.token_logprobs(whole[:, 3:4], t).logprob.tolist() == [0.0] * 4
    assert float(flat.abs().sum()) == 0.0
