"""What a step of beam search may not write over: the parents that the moving of states reads.  Every refusal comes before a launch."""
from array import array

import pytest

from paper_2002_09539_amd import binding as B

A = 0x7F0000000000      # 256-byte aligned stand-in for device addresses; never dereferenced


def refused(call, part):
    with pytest.raises(B.OlsError) as e:
        call()
    assert e.value.code == B.OLS_EINVAL and part in str(e.value), str(e.value)


def reorder(parent, dst, src, row_bytes=40, n=2, at=1, batch=2, beams=3, beam=40, batch_stride=120):
    """n tensors, all of them apart but number `at`."""
    far = [A + (1 << 30) + (i << 20) for i in range(2 * n)]
    far[at], far[n + at] = src, dst
    arrays = [array("Q", far[:n]), array("Q", far[n:])] + [array("q", [v] * n) for v in (row_bytes, batch_stride, beam, batch_stride, beam)]
    B.ols_beam_reorder(n, *[a.buffer_info()[0] for a in arrays], batch, beams, beams, parent, None)


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("parent", [A, A + 4, A - 20, A + 116, A + 236])
def test_parents_among_what_is_written(parent, at):
    """24 bytes of parents, states of 2 x 120 bytes from A on."""
    refused(lambda: reorder(parent, A, A, at=at), "parents")                    # in place
    refused(lambda: reorder(parent, A, A + 4096, at=at), "parents")             # apart


def test_parents_in_the_last_of_rows_that_are_apart():
    refused(lambda: reorder(A + 1000 + 2 * 100 + 12, A, A, row_bytes=16, beam=100, batch_stride=1000), "parents")
    refused(lambda: reorder(A + 80, A, A, row_bytes=16, beam=100, batch_stride=1000), "parents")        # reach into the second row from the gap before it
