"""A hypothesis' candidates come in the order of its logits also where their values, in 64 bits, are one number, and however its row is cut
into parts: scores that are large beside the logits, and logits that are tiny beside the score."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _best(z, k):
    """The places of the k largest of one row, ties to the lower."""
    return torch.sort(z.cpu().double(), descending=True, stable=True).indices[:k].tolist()


def _check(z, score, beams):
    from paper_2002_09539_amd import operators as ops
    b = ops.beam_select(z, torch.full(z.shape[:2], score, device="cuda"), beams=beams)
    for r in range(z.shape[0]):
        want = [(0, t) for t in _best(z[r, 0], beams)]
        assert list(zip(b.parent[r].tolist(), b.token[r].tolist())) == want
    many = ops.beam_select(z[:1].repeat(600, 1, 1), torch.full((600, z.shape[1]), score, device="cuda"), beams=beams)
    assert torch.equal(many.token, b.token[:1].expand(600, beams)) and torch.equal(many.parent, b.parent[:1].expand(600, beams))


# lists of the merge: one for each lane, some for each, and more than a lane's registers or than LDS holds
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("have,vocab,beams", [(1, 20001, 4), (2, 40003, 8), (1, 100001, 32), (8, 60001, 5)])
def test_scores_that_swallow_the_logits(have, vocab, beams, dtype):
    """All ranks of all hypotheses are one number: the first hypothesis' best, most of which lie in its last part."""
    z = torch.randn(2, have, vocab, generator=torch.Generator(device="cuda").manual_seed(vocab), device="cuda")
    z[:, :, vocab - 3:] += 20.0
    z[:, :, 7] = 9.0
    z[1, :, :] = 0.0
    z[1, :, vocab - 2] = 1.0
    z[1, :, vocab // 2] = 1.0                               # equal ones of two parts: the lower token
    for score in (-1e30, -3e38):
        _check(z.to(dtype), score, beams)


@pytest.mark.parametrize("have,vocab", [(17, (1 << 20) + 5), (32, 20011)])
def test_more_lists_than_registers_hold(have, vocab):
    from paper_2002_09539_amd import operators as ops
    z = torch.randn(1, have, vocab, generator=torch.Generator(device="cuda").manual_seed(vocab), device="cuda")
    z[:, :, vocab - 3:] += 20.0
    for beams in (9, 32):
        b = ops.beam_select(z, torch.full((1, have), -1e30, device="cuda"), beams=beams)
        assert b.parent[0].tolist() == [0] * beams and b.token[0].tolist() == _best(z[0, 0], beams)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,beams", [(20001, 4), (100001, 32)])
def test_logits_that_vanish_beside_the_score(vocab, beams, dtype):
    """Different logits of 1e-30 and less, whose differences a score of -3 does not hold."""
    z = torch.rand(2, 1, vocab, generator=torch.Generator(device="cuda").manual_seed(vocab), device="cuda") * 1e-30
    z[:, :, vocab - 5:] += 1e-30
    _check(z.to(dtype), -3.0, beams)


def test_ended_hypotheses_among_them():
    """One that has ended has no logits: it comes before or behind all that a hypothesis of the same rank offers, by its number."""
    from paper_2002_09539_amd import operators as ops
    z = torch.randn(1, 3, 40003, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    z[:, :, 40000:] += 20.0
    z[0, 1] = float("nan")
    finished = torch.tensor([[False, True, False]], device="cuda")
    b = ops.beam_select(z, torch.full((1, 3), -1e30, device="cuda"), beams=8, finished=finished, eos=2)
    assert b.parent[0].tolist() == [0] * 8 and b.token[0].tolist() == _best(z[0, 0], 8)
    z[0, 0, 5:] = float("-inf")                             # five candidates, then the one that has ended, then the third's
    b = ops.beam_select(z, torch.full((1, 3), -1e30, device="cuda"), beams=8, finished=finished, eos=2)
    assert b.parent[0].tolist() == [0] * 5 + [1, 2, 2]
    assert b.token[0].tolist() == _best(z[0, 0], 5) + [2] + _best(z[0, 2], 2)


@pytest.mark.parametrize("penalty", [0.0, 1.0, 0.7])
@pytest.mark.parametrize("top", [0.0, 255.0])
def test_the_smallest_differences_that_values_hold(top, penalty):
    """Logits from 2^-16 on, one unit in the last place apart, under the largest score that still tells all of them apart, and beyond."""
    from paper_2002_09539_amd import operators as ops
    vocab, beams = 40003, 9
    z = 2.0 ** -16 * (1 + torch.randperm(vocab, generator=torch.Generator().manual_seed(1)).float() * 2.0 ** -23)
    z[20000] = top
    z = z.cuda()[None, None]
    for score in (-1000.0, -1013.0, -1100.0, 900.0):
        b = ops.beam_select(z, torch.full((1, 1), score, device="cuda"), beams=beams, length=torch.full((1, 1), 6, dtype=torch.int32, device="cuda"), length_penalty=penalty)
        assert b.token[0].tolist() == _best(z[0, 0], beams)
