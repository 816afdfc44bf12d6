"""The order of a beam search's candidates where it hangs on equal numbers: equal quotients of hypotheses of different lengths.

Scores are whole multiples of a few bits, so that quotients are exact; what is compared are whole numbers."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _ended(scores, lengths, penalty):
    """The order in which hypotheses that have all ended come out: their parents."""
    batch, have = scores.shape
    z = torch.zeros(batch, have, 50, device="cuda")
    b = _ops().beam_select(z, scores.cuda(), finished=torch.ones(batch, have, dtype=torch.bool, device="cuda"), length=lengths.cuda(), eos=1, length_penalty=penalty)
    assert bool((b.token == 1).all()) and torch.equal(b.score.cpu(), scores.gather(1, b.parent.cpu().long()))
    return b.parent.cpu()


@pytest.mark.parametrize("penalty,power", [(1.0, lambda n: n), (2.0, lambda n: n * n), (3.0, lambda n: n ** 3), (-1.0, lambda n: 1.0 / n), (0.0, lambda n: 1)])
def test_equal_quotients_of_different_lengths(penalty, power):
    """Sets of 32 hypotheses with one average: places go by number alone."""
    g = torch.Generator().manual_seed(int(10 * penalty) + 100)
    lengths = torch.randint(1, 60, (300, 32), generator=g, dtype=torch.int32)
    if penalty < 0:
        lengths = 1 << torch.randint(0, 12, (300, 32), generator=g, dtype=torch.int32)      # whose quotients fp32 scores can hold
    averages = -torch.randint(1, 9, (300, 1), generator=g).double() / 8 - 1
    scores = (averages * lengths.double().apply_(power)).float()
    assert bool((scores.double() == averages * lengths.double().apply_(power)).all())
    assert torch.equal(_ended(scores, lengths, penalty), torch.arange(32, dtype=torch.int32).expand(300, 32))


def test_equal_quotients_by_the_root_of_the_length():
    roots = torch.randint(1, 100, (200, 16), generator=torch.Generator().manual_seed(1))
    scores = -1.25 * roots.float()
    assert torch.equal(_ended(scores, (roots * roots).int(), 0.5), torch.arange(16, dtype=torch.int32).expand(200, 16))


@pytest.mark.parametrize("penalty,root,power", [(0.25, 4, 1), (0.75, 4, 3), (1.5, 2, 3), (2.125, 8, 17), (0.0625, 16, 1), (-0.5, 2, -1)])
def test_equal_quotients_by_other_roots(penalty, root, power):
    """Lengths n ** root, scores avg * n ** power: whole numbers of few bits, or powers of two where the power is negative or large."""
    bases = torch.tensor([[1, 2, 4, 1, 2, 4, 2, 1]] if power < 0 or power > 4 else [[3, 1, 2, 3, 5, 7, 6, 2]] if root < 16 else [[1, 2, 3, 2, 1, 3, 1, 2]])
    for average in (-1.25, -0.875):
        for order in range(8):
            n = bases.roll(order, 1)
            scores = (average * n.double() ** power).float()
            assert torch.equal(_ended(scores, (n ** root).int(), penalty), torch.arange(8, dtype=torch.int32)[None])


def test_the_longer_of_two_that_are_equal():
    """The pair of the smallest numbers, in both orders, and one unit in the last place to either side."""
    below, above = torch.nextafter(torch.tensor(-3.75), torch.tensor(-math.inf)), torch.nextafter(torch.tensor(-3.75), torch.tensor(0.0))
    scores = torch.tensor([[-3.75, -1.25], [-1.25, -3.75], [float(below), -1.25], [float(above), -1.25]])
    lengths = torch.tensor([[3, 1], [1, 3], [3, 1], [3, 1]], dtype=torch.int32)
    assert _ended(scores, lengths, 1.0).tolist() == [[0, 1], [0, 1], [1, 0], [0, 1]]


def test_a_length_of_none_counts_as_one():
    scores, lengths = torch.tensor([[-2.5, -1.25, -1.25]]), torch.tensor([[2, 0, 1]], dtype=torch.int32)
    assert _ended(scores, lengths, 1.0).tolist() == [[0, 1, 2]]


@pytest.mark.parametrize("change", [dict(eos=(1 << 32) + 3), dict(eos=-(1 << 32) + 3), dict(eos=1 << 31), dict(beams=(1 << 32) + 2), dict(beams=-(1 << 32) + 2)])
def test_numbers_that_the_boundary_does_not_hold(change):
    """Modulo 2^32 they would be a token or a number of hypotheses."""
    from paper_2002_09539_amd import binding as B
    with pytest.raises(B.OlsError):
        _ops().beam_select(torch.zeros(1, 2, 8, device="cuda"), torch.zeros(1, 2, device="cuda"), **change)
    b = _ops().beam_select(torch.zeros(1, 2, 8, device="cuda"), torch.zeros(1, 2, device="cuda"), eos=-(1 << 31))
    assert not bool(b.finished.any())
