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


# ---- results of the choice --------------------------------------------------------------------------------------------
PLACES = dict(logits=0, score=1, finished=2, length=3, new_score=4, token=5, parent=6, new_length=7, new_finished=8, ws=9)
RESULTS = {"new_score": "score", "new_length": "length", "new_finished": "finished", "token": None, "parent": None}


def select(in_beams=3, beams=3, **change):
    """2 requests of 3 hypotheses, every array a megabyte from the next but for those in `change`."""
    b = B.ols_beam()
    b.dtype, b.in_beams, b.beams, b.eos, b.batch, b.vocab, b.batch_stride, b.beam_stride, b.length_penalty = B.OLS_F32, in_beams, beams, 2, 2, 100, 100 * in_beams, 100, 1.0
    b.ws_bytes = 1 << 18
    for name, i in PLACES.items():
        setattr(b, name, change.get(name, A + (i << 20)))
    B.ols_beam_select(b, None)


def place(name):
    return A + (PLACES[name] << 20)


@pytest.mark.parametrize("result", list(RESULTS))
@pytest.mark.parametrize("other", ["score", "finished", "length", "ws"])
def test_results_of_the_choice_on_what_it_reads(result, other):
    """The choice of one request is written while another's hypotheses are read."""
    beams = 4 if RESULTS[result] == other else 3             # where the shapes are one it may take the place of what it follows
    refused(lambda: select(beams=beams, **{result: place(other)}), "overlap")
    if result != "new_finished":
        refused(lambda: select(beams=3, **{result: place(other) + 4}), "overlap")


@pytest.mark.parametrize("a,b", [("new_score", "token"), ("token", "parent"), ("parent", "new_length"), ("new_score", "new_finished"), ("new_finished", "new_length")])
def test_results_of_the_choice_on_each_other(a, b):
    refused(lambda: select(**{b: place(a)}), "overlap")
    refused(lambda: select(**{b: place(a) + 4}), "overlap")         # the shortest has six bytes
