"""States that share memory with what else a call reads or writes: taken where that is sound, refused otherwise."""
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def test_the_parents_are_not_moved():
    ops = _ops()
    parent = torch.tensor([[1, 0, 2], [2, 2, 0]], dtype=torch.int32, device="cuda")
    s, before = torch.randn(2, 3, 700, device="cuda"), parent.clone()
    start = s.clone()
    for call in (lambda: ops.beam_reorder([s, parent], parent), lambda: ops.beam_reorder([parent], parent), lambda: ops.beam_reorder([before], parent, out=[parent]),
                 lambda: ops.beam_reorder([s, parent.view(torch.uint8).view(2, 3, 4)], parent)):
        with pytest.raises(B.OlsError, match="parents"):
            call()
    assert torch.equal(parent, before) and torch.equal(s, start)
    other = torch.empty_like(parent)
    ops.beam_reorder([s, parent], parent, out=[torch.empty_like(s), other])          # read alone
    assert torch.equal(other, parent.gather(1, parent.long()))


def test_parents_between_the_rows_of_a_state():
    ops = _ops()
    buf = torch.arange(120, dtype=torch.int32, device="cuda").view(2, 3, 20)
    parent = buf[0, 0, 10:16].view(2, 3)
    parent.copy_(torch.tensor([[1, 0, 2], [2, 2, 0]]))
    want = buf.clone()
    want[:, :, :10] = buf[torch.arange(2, device="cuda")[:, None], parent.long()][:, :, :10]
    ops.beam_reorder([buf[:, :, :10]], parent)
    assert torch.equal(buf, want)


def test_parents_that_are_copied_first_may_be_moved():
    """Columns of a wider array are no contiguous parents: the call reads a copy of them."""
    ops = _ops()
    wide = torch.tensor([[1, 0, 2, 9], [2, 2, 0, 9]], dtype=torch.int32, device="cuda")
    parent = wide[:, :3]
    want = parent.gather(1, parent.long())
    ops.beam_reorder([parent], parent)
    assert torch.equal(wide[:, :3], want) and bool((wide[:, 3] == 9).all())


def test_a_state_that_is_read_twice_does_not_move_in_place():
    """Its other copy would be taken from what has moved already, or not, as workgroups come."""
    ops = _ops()
    parent = torch.tensor([[1, 0, 2], [2, 2, 0]], dtype=torch.int32, device="cuda")
    a, b, c = (torch.randn(2, 3, 5000, device="cuda") for _ in range(3))
    start = a.clone()
    for states, out in (([a, a], [b, a]), ([a, a], [a, b]), ([a, c, a], [b, c, a])):
        with pytest.raises(B.OlsError, match="another state"):
            ops.beam_reorder(states, parent, out=out)
    assert torch.equal(a, start)
    rows = torch.arange(2, device="cuda")[:, None]
    ops.beam_reorder([a, a], parent, out=[b, c])
    assert torch.equal(b, a[rows, parent.long()]) and torch.equal(c, b)
    ops.beam_reorder([a, c], parent, out=[b, c])            # one in place, one apart
    assert torch.equal(a, start) and torch.equal(c, b[rows, parent.long()])
