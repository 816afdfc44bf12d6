"""A step of beam search and the moving of states, against the candidates of 64 bits put in order.

Whole numbers have to be equal.  Scores are sums of fp64 values, rounded once (2^-24), of a logarithm whose sum of fp32 exponentials has a
relative error of a few 2^-24: 1e-6 absolute and 2^-23 of the score."""
import math

import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def want(z, score, beams, finished, length, eos, penalty):
    """Rows of (score, token, parent, finished, length) for one request; z double [hypotheses][vocab]."""
    have = z.shape[0]
    rows, poisoned = [], False
    for i in range(have):
        s, n = float(score[i]), (0 if length is None else int(length[i]))
        if s == -math.inf:
            continue
        ended = finished is not None and bool(finished[i])
        if math.isnan(s) or s == math.inf or (not ended and bool((torch.isnan(z[i]) | (z[i] == math.inf)).any())):
            poisoned = True
            continue
        if ended:
            rows.append((s / max(n, 1) ** penalty, i, 0, s, eos, True, n))
            continue
        top = float(z[i].max())
        if top == -math.inf:
            continue
        lse = math.log(float(torch.exp(z[i] - top).sum()))
        best = torch.argsort(-z[i], stable=True)[:beams]
        for t in best.tolist():
            if float(z[i, t]) > -math.inf:
                v = s + (float(z[i, t]) - top - lse)
                rows.append((v / max(n + 1, 1) ** penalty, i, t, v, t, eos >= 0 and t == eos, n + 1))
    rows.sort(key=lambda r: (-r[0], r[1], r[2]))
    rows = [] if poisoned else rows[:beams]
    out = [(v, t, i, f, n) for _, i, _, v, t, f, n in rows]
    for k in range(len(out), beams):
        slot = k if k < have else 0
        out.append((math.nan if poisoned else -math.inf, -1, slot, False, 0 if length is None else int(length[slot])))
    return out


def check(z, score, beams=None, finished=None, length=None, eos=-1, penalty=0.0):
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    k = beams or z.shape[1]
    b = _ops().beam_select(z.cuda(), dev(score), beams=beams, finished=dev(finished), length=dev(length), eos=eos, length_penalty=penalty)
    assert b.score.shape == (z.shape[0], k) and b.token.dtype == torch.int32 and b.finished.dtype == torch.bool
    for r in range(z.shape[0]):
        rows = want(z[r].double(), score[r], k, None if finished is None else finished[r], None if length is None else length[r], eos, penalty)
        for j, (v, t, i, f, n) in enumerate(rows):
            got = float(b.score[r, j])
            assert (int(b.token[r, j]), int(b.parent[r, j]), bool(b.finished[r, j])) == (t, i, f), (r, j, v, got)
            assert got == v or (math.isnan(v) and math.isnan(got)) or abs(got - v) <= 1e-6 + 2.0 ** -23 * abs(v), (r, j, got, v)
            if length is not None:
                assert int(b.length[r, j]) == n
    assert (b.length is None) == (length is None)
    return b


def inputs(seed, batch, have, vocab, dtype, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(batch, have, vocab, generator=g) * 2.5
    if masked:
        z[torch.rand(batch, have, vocab, generator=g) < masked] = -math.inf
    score = torch.randn(batch, have, generator=g) - 20
    length = torch.randint(0, 40, (batch, have), generator=g, dtype=torch.int32)
    finished = torch.rand(batch, have, generator=g) < 0.25
    return z.to(dtype), score, finished, length


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,have,vocab,beams", [(1, 1, 1, 1), (1, 1, 50, 4), (2, 3, 2, 7), (3, 4, 1000, 4), (1, 32, 77, 32), (2, 5, 4097, 5), (1, 4, 32000, 4), (7, 5, 3203, 2),
                                                    (130, 4, 300, 4), (40, 16, 2500, 16)])
def test_selection(batch, have, vocab, beams, dtype):
    z, score, finished, length = inputs(batch * vocab + have, batch, have, vocab, dtype)
    check(z, score, beams)
    check(z, score, beams, finished=finished, eos=min(2, vocab - 1))
    check(z, score, beams, finished=finished, length=length, eos=0, penalty=0.7)
    check(z, score, beams, length=length, penalty=-0.5)


@pytest.mark.parametrize("dtype,batch,have,vocab", [(F32, 1, 32, 20011), (BF16, 2, 31, 9000), (F32, 1, 3, (1 << 20) + 5), (F32, 1, 17, (1 << 20) + 5), (F32, 1, 2, 70001), (BF16, 1, 3, 140001), (BF16, 128, 4, 20011), (BF16, 64, 8, 70001), (F32, 64, 8, 40001), (BF16, 64, 8, 33001)])
def test_long_rows(dtype, batch, have, vocab):
    """Rows in parts, and each size of workgroup; some requests of the many are looked at."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn(batch, have, vocab, generator=g, device="cuda") * 2.5).to(dtype)
    score = torch.randn(batch, have, generator=torch.Generator().manual_seed(1)) - 5
    b = _ops().beam_select(z, score.cuda())
    for r in sorted({0, batch // 2, batch - 1}):
        for j, (v, t, i, _, _) in enumerate(want(z[r].cpu().double(), score[r], have, None, None, -1, 0.0)):
            assert (int(b.token[r, j]), int(b.parent[r, j])) == (t, i)
            assert abs(float(b.score[r, j]) - v) <= 1e-6 + 2.0 ** -23 * abs(v)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_ends_and_empty_places(dtype):
    z, score, finished, length = inputs(5, 9, 4, 600, dtype, masked=0.4)
    score[0, 1:] = -math.inf                    # a search begins
    score[1] = -math.inf                        # no hypothesis at all
    z[2] = -math.inf                            # nothing may follow
    finished[2] = False
    z[3] = -math.inf
    z[3, 1, 5:7] = 0.25                         # two candidates for four places
    finished[3] = torch.tensor([True, False, False, False])
    finished[4] = True                          # all have ended
    z[4] = math.nan                             # and are not read
    z[5, 2] = math.nan                          # a hypothesis that is no hypothesis is not read either
    score[5, 2] = -math.inf
    z[6] = torch.finfo(dtype).min
    z[7, :, 3] = 50.0                           # the end wins everywhere
    length[8] = 0
    for eos in (3, -1):
        check(z, score, finished=finished, length=length, eos=eos, penalty=1.0)
        check(z, score, finished=finished, eos=eos)
        check(z, score, beams=7, finished=finished, length=length, eos=eos)


@pytest.mark.parametrize("parts", [False, True])
def test_ties_go_to_the_lower_hypothesis_and_token(parts):
    vocab = 20000 if parts else 500
    z = torch.zeros(1 if parts else 600, 3, vocab)
    z[:, :, 100] = 1.0
    z[:, :, 40] = 1.0
    score = torch.zeros(z.shape[0], 3)
    b = check(z[:2], score[:2]) if not parts else check(z, score)
    b = _ops().beam_select(z.cuda(), score.cuda(), beams=8)
    assert b.token[0].tolist() == [40, 100, 40, 100, 40, 100, 0, 1] and b.parent[0].tolist() == [0, 0, 1, 1, 2, 2, 0, 0]
    assert torch.equal(b.token, b.token[:1].expand_as(b.token))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [3, 8, 9, 32])
def test_best_that_one_lane_holds(k, dtype):
    """The best all side by side, in one lane's registers and its neighbours', and the same value everywhere else: lists longer than their room."""
    vocab = 32768 if dtype == BF16 else 16384
    z = torch.full((2, 1, vocab), -3.0)
    z[0, 0, 4096: 4096 + 40] = torch.arange(40).float() / 8
    z[1, 0, ::1] = torch.where(torch.arange(vocab) % 3 == 0, 2.0, -5.0)
    score = torch.zeros(2, 1)
    z = z.to(dtype)
    check(z, score, beams=k)
    many = _ops().beam_select(z.repeat(300, 1, 1).cuda(), score.repeat(300, 1).cuda(), beams=k)        # whole rows in a workgroup
    few = _ops().beam_select(z.cuda(), score.cuda(), beams=k)
    assert torch.equal(many.token, few.token.repeat(300, 1))
    assert float((many.score - few.score.repeat(300, 1)).abs().max()) <= 2e-6 + 2.0 ** -22 * 9      # each within the tolerance above: sums of other parts


def test_what_is_not_finite_stays_in_its_request():
    z, score, _, length = inputs(6, 6, 3, 300, F32)
    z[1, 2, 17] = math.nan
    z[2, 0, 299] = math.inf
    score[3, 1] = math.nan
    score[4, 1] = math.inf
    b = check(z, score, length=length, penalty=0.5)
    assert bool(torch.isnan(b.score[1:5]).all()) and not bool(torch.isnan(b.score[[0, 5]]).any())
    z[:] = 0.0
    z[0, 0, 1] = math.nan
    check(z[:1].repeat(600, 1, 1)[:3], score[:1].repeat(3, 1))


def test_strides_streams_and_capture():
    ops = _ops()
    z, score, finished, length = (t.cuda() for t in inputs(7, 4, 3, 900, BF16))
    plain = ops.beam_select(z, score, finished=finished, length=length, eos=1, length_penalty=0.6)
    wide = torch.full((3, 4, 1000), math.nan, dtype=BF16, device="cuda")
    wide[:, :, 33:933] = z.transpose(0, 1)
    apart = ops.beam_select(wide[:, :, 33:933].transpose(0, 1), score.t().contiguous().t(), finished=finished, length=length, eos=1, length_penalty=0.6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = ops.beam_select(z, score, finished=finished, length=length, eos=1, length_penalty=0.6)
    side.synchronize()
    for b in (apart, other):
        assert all(torch.equal(x, y) for x, y in zip(b, plain))
    shared = ops.beam_select(z[:1, :1].expand(4, 3, 900), score)          # one row of logits for all
    assert torch.equal(shared.token, ops.beam_select(z[:1, :1].expand(4, 3, 900).contiguous(), score).token)
    state = torch.randn(4, 3, 50, device="cuda")
    start = state.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b = ops.beam_select(z, score, finished=finished, length=length, eos=1, length_penalty=0.6)
        ops.beam_reorder([state], b.parent)
    for seed in (8, 9, 10):
        z.copy_(inputs(seed, 4, 3, 900, BF16)[0])
        state.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        eager = ops.beam_select(z, score, finished=finished, length=length, eos=1, length_penalty=0.6)
        assert all(torch.equal(x, y) for x, y in zip(b, eager))
        assert torch.equal(state, start[torch.arange(4, device="cuda")[:, None], eager.parent.long()])


# ---- states -----------------------------------------------------------------------------------------------------------
def moved(t, parent):
    old, new = t.clone(), t.clone()
    for r in range(parent.shape[0]):
        for i in range(parent.shape[1]):
            p = int(parent[r, i])
            if 0 <= p < t.shape[1]:
                new[r, i] = old[r, p]
    return new


@pytest.mark.parametrize("beams", [1, 3, 4, 8, 9, 16, 17, 32])
def test_states_in_place_and_apart(beams):
    ops = _ops()
    g = torch.Generator().manual_seed(beams)
    batch = 5
    parent = torch.randint(0, beams, (batch, beams), generator=g, dtype=torch.int32)
    parent[0] = torch.arange(beams)                        # nothing moves
    parent[1] = beams - 1 - torch.arange(beams)            # turned round
    if beams > 2:
        parent[2, 1], parent[2, 2] = -1, beams             # left as they are
    states = [torch.randint(-100, 100, (batch, beams, n), generator=g).to(d) for n, d in ((1, torch.int8), (3, torch.int16), (17, torch.int32), (1, torch.int64), (5000, torch.uint8),
                                                                                          (0, torch.float32))]
    states += [torch.randn(batch, beams, 3, 11, generator=g), torch.randn(batch, beams, generator=g).bfloat16(), torch.randn(batch, beams, 4097, generator=g).bfloat16()]
    want_all = [moved(t, parent) for t in states]
    here = [t.cuda() for t in states]
    back = ops.beam_reorder(here, parent.cuda())
    assert all(x is y for x, y in zip(back, here))
    for x, w in zip(here, want_all):
        assert torch.equal(x.cpu(), w)
    src = [t.cuda() for t in states]
    out = [torch.zeros_like(t) for t in src]
    ops.beam_reorder(src, parent.cuda(), out=out)
    for x, s, w in zip(out, states, want_all):
        keep = ((parent >= 0) & (parent < beams)).view(batch, beams, *([1] * (s.dim() - 2)))
        assert torch.equal(x.cpu(), torch.where(keep, w, torch.zeros_like(w)))
    assert all(torch.equal(x.cpu(), s) for x, s in zip(src, states))


def test_states_of_more_or_fewer_places_and_slices():
    ops = _ops()
    cache = torch.randn(3, 2, 40, 6, device="cuda")
    parent = torch.tensor([[0, 1, 1, 0, 1], [1, 1, 1, 1, 1], [0, 0, 0, 0, 1]], dtype=torch.int32, device="cuda")
    out = torch.full((3, 5, 40, 6), 9.0, device="cuda")
    ops.beam_reorder([cache[:, :, :13]], parent, out=[out[:, :, :13]])
    rows = torch.arange(3, device="cuda")[:, None]
    assert torch.equal(out[:, :, :13], cache[rows, parent.long()][:, :, :13]) and bool((out[:, :, 13:] == 9).all())
    few = torch.tensor([[1], [0], [1]], dtype=torch.int32, device="cuda")
    one = torch.empty(3, 1, 40, 6, device="cuda")
    ops.beam_reorder([cache], few, out=[one])
    assert torch.equal(one, cache[rows, few.long()])
    many = [torch.randn(3, 2, n + 1, device="cuda") for n in range(130)]         # more tensors than a launch takes
    swap = torch.tensor([[1, 0]] * 3, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in many]
    ops.beam_reorder(many, swap)
    assert all(torch.equal(t, b.flip(1)) for t, b in zip(many, before))
    across = torch.randn(2, 3, 8, device="cuda").transpose(0, 1)                  # hypotheses in front of requests
    old = across.clone()
    ops.beam_reorder([across], swap)
    assert torch.equal(across, old.flip(1))
    assert ops.beam_reorder([], swap) == []


def test_refusals():
    ops = _ops()
    z, score, finished, length = (t.cuda() for t in inputs(9, 2, 3, 40, F32))
    parent = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    s = torch.zeros(2, 3, 8, device="cuda")
    two = torch.zeros(2, 2, 3, 8, device="cuda")
    for call in (lambda: ops.beam_select(z[0], score), lambda: ops.beam_select(z, score[:, :2]), lambda: ops.beam_select(z, score.double()),
                 lambda: ops.beam_select(z, score, beams=33), lambda: ops.beam_select(z, score, beams=0), lambda: ops.beam_select(z.double(), score),
                 lambda: ops.beam_select(z.transpose(1, 2), score), lambda: ops.beam_select(z, score, length_penalty=1.0),
                 lambda: ops.beam_select(z, score, length=length, length_penalty=math.nan), lambda: ops.beam_select(z, score, finished=finished.int()),
                 lambda: ops.beam_select(z, score.cpu()), lambda: ops.beam_select(z, score, length=length.long()), lambda: ops.beam_select(z[:, :, :0], score),
                 lambda: ops.beam_reorder([s], parent.long()), lambda: ops.beam_reorder([s], parent[:, :2]), lambda: ops.beam_reorder([s[:1]], parent),
                 lambda: ops.beam_reorder([s, s], parent), lambda: ops.beam_reorder([s], parent, out=[s[:, :, :4]]), lambda: ops.beam_reorder([s], parent, out=[]),
                 lambda: ops.beam_reorder([s.transpose(0, 2)], parent), lambda: ops.beam_reorder([s[:, :, ::2]], parent), lambda: ops.beam_reorder([s[0]], parent),
                 lambda: ops.beam_reorder([two[0], two[1]], parent, out=[two[1], two[0]]), lambda: ops.beam_reorder([s[:1, :1].expand(2, 3, 8)], parent),
                 lambda: ops.beam_reorder([s], parent, out=[torch.zeros(2, 1, 8, device="cuda").expand(2, 3, 8)]),
                 lambda: ops.beam_reorder([s.view(-1)[:24].view(1, 3, 8)], parent[:1], out=[s.view(-1)[8:32].view(1, 3, 8)]),
                 lambda: ops.beam_reorder([s.cpu()], parent)):
        with pytest.raises(B.OlsError):
            call()
