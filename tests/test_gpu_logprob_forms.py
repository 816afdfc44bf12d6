"""Targets that cannot occur: what their log probabilities and gradients are, in both ways to the gradient."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [7, 5000, 140_000])
def test_a_target_of_minus_infinity(dtype, vocab):
    """logprob -inf; the gradient is the formula's, d_logprob ([j = target] - p_j), with p = 0 at the target: good to the rounding of p
    (2e-5) and of the type.  In a row of nothing else it is zero."""
    z = torch.randn(3, vocab, generator=torch.Generator(device="cuda").manual_seed(vocab), device="cuda").to(dtype)
    z[0, 4] = -math.inf
    z[1] = -math.inf
    z[2, 4:] = -math.inf
    t = torch.full((3,), 4, dtype=torch.int32, device="cuda")
    up = torch.tensor([0.75, 0.5, -1.5], device="cuda")
    r, d = _ops().token_logprobs_with_grad(z, t, up)
    later = _ops().token_logprobs_grad(z, t, r, up)
    assert r.logprob.tolist() == [-math.inf] * 3
    p = torch.softmax(z.double(), 1)
    want = -up.double()[:, None] * p
    want[:, 4] = up.double()
    want[1] = 0.0
    for got in (d, later):
        assert got[:, 4].tolist() == [0.75, 0.0, -1.5]
        assert ((got.double() - want).abs() <= 2e-5 + 2.0 ** -8 * want.abs()).all()
