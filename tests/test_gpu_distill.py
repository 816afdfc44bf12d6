"""Distillation from a teacher's top logits, with the likelihood of a given token, and the gradient, against 64 bits.

Tolerances.  In fp32 the sums have relative errors of a few 2^-24 (positive terms in short partial sums, each exponential good to 2
units in the last place plus 2^-24 of its argument's size); ATOL = 4e-6 holds ten times that in a logarithm, for |z - m| / T <= 60.  A loss
has at most two such logarithms (of the sum and of the rest's), so 2 ATOL T^2, and is rounded once.  A gradient entry is probabilities
of relative error 1e-5 times T d_loss or d_logprob, plus the storage rounding: 2e-5 of those factors."""
import math

import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ATOL, GTOL = 4e-6, 2e-5


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def want_row(z, value, index, target, T, rest, g_loss, g_hard):
    """Loss, log probability and gradient of one row, from the formulas in 64 bits."""
    vocab = z.numel()
    entries = [(int(i), float(v)) for i, v in zip(index, value) if 0 <= int(i) < vocab]
    has = 0 <= target < vocab
    bad = bool(torch.isnan(z).any() or (z == math.inf).any())
    bad_list = any(math.isnan(v) or v == math.inf for _, v in entries)
    if bad or bad_list:
        lp = 0.0
        if has:
            lp = math.nan if bad else float(torch.log_softmax(z, 0)[target])
        return math.nan, lp, torch.full((vocab,), math.nan, dtype=torch.float64)
    if rest:
        q = [math.exp(v) for _, v in entries]
        log_q = [v for _, v in entries]
        q_r = max(0.0, 1.0 - math.fsum(q)) if entries else 0.0
    else:
        top = max([v for _, v in entries], default=-math.inf)
        e = [math.exp((v - top) / T) if top > -math.inf else 0.0 for _, v in entries]
        total = math.fsum(e)
        q = [x / total if total else 0.0 for x in e]
        log_q = [(v - top) / T - math.log(total) if total else 0.0 for _, v in entries]
        q_r = 0.0
    if bool((z == -math.inf).all()):
        return (math.inf if any(x > 0 for x in q) else 0.0), (-math.inf if has else 0.0), torch.zeros(vocab, dtype=torch.float64)
    u = (z - z.max()) / T
    log_p = u - torch.logsumexp(u, 0)
    p = log_p.exp()
    loss = math.fsum(x * (l - float(log_p[i])) for x, l, (i, _) in zip(q, log_q, entries) if x > 0)
    member = torch.zeros(vocab, dtype=torch.bool)
    for i, _ in entries:
        member[i] = True
    weight = math.fsum(q)
    grad = p * 0
    log_left = torch.logsumexp(torch.where(member, -math.inf, log_p), 0) if not bool(member.all()) else torch.tensor(-math.inf, dtype=torch.float64)
    if q_r > 0 and float(log_left) > -math.inf:
        loss += q_r * (math.log(q_r) - float(log_left))
        weight += q_r
        left = torch.where(member, -math.inf, u)                  # p / p_r against the others' own largest: -3e38 holds no logarithm beside it
        grad = grad - q_r * torch.softmax(left - left.max(), 0)
    grad = grad + weight * p
    for x, (i, _) in zip(q, entries):
        grad[i] -= x
    grad = grad * (T * g_loss)
    row = z - z.max()
    lsm = row - torch.logsumexp(row, 0)
    lp = 0.0
    if has:
        lp = float(lsm[target])
        grad = grad - g_hard * lsm.exp()
        grad[target] += g_hard
    return T * T * loss, lp, grad


def lists(seed, rows, vocab, k, rest, missing=0.1):
    """Indices without repetition in a row, some of them none, and values that rest's mass stays positive with."""
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(vocab, generator=g)[:k] if k <= vocab else torch.randint(0, vocab, (k,), generator=g) for _ in range(rows)])
    value = torch.randn(rows, k, generator=g) * 2
    if rest:
        value = torch.log_softmax(torch.cat([value, torch.zeros(rows, 1)], 1), 1)[:, :k]
    index[torch.rand(rows, k, generator=g) < missing] = -1
    return value.float().contiguous(), index.to(torch.int32).contiguous()


def logits(seed, rows, vocab, dtype, masked=0.0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * spread
    if masked:
        z[torch.rand(rows, vocab, generator=g) < masked] = -math.inf
    return z.to(dtype)


def check(z, value, index, t, T, rest, separate=True, in_place=True):
    ops = _ops()
    rows, vocab = z.shape
    g = torch.Generator().manual_seed(rows + vocab)
    gl, gh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    want = [want_row(z[r].double(), value[r], index[r], -1 if t is None else int(t[r]), T, rest, float(gl[r]), float(gh[r])) for r in range(rows)]
    zd, vd, xd, td = z.cuda(), value.cuda(), index.cuda(), None if t is None else t.cuda()
    hard = None if t is None else gh.cuda()
    calls = []
    first = ops.distill_loss(zd, vd, xd, targets=td, temperature=T, rest=rest)
    assert torch.equal(zd.cpu().view(torch.int16 if z.dtype == BF16 else torch.int32), z.view(torch.int16 if z.dtype == BF16 else torch.int32))
    r, d = ops.distill_loss_with_grad(zd, vd, xd, gl.cuda(), targets=td, d_logprob=hard, temperature=T, rest=rest)
    calls.append((r, d))
    if separate:
        calls.append((first, ops.distill_loss_grad(zd, vd, xd, first, gl.cuda(), targets=td, d_logprob=hard, temperature=T, rest=rest)))
    if in_place:
        z2 = zd.clone()
        r2, d2 = ops.distill_loss_with_grad(z2, vd, xd, gl.cuda(), targets=td, d_logprob=hard, temperature=T, rest=rest, out=z2)
        assert d2 is z2
        calls.append((r2, d2))
        if separate:
            z3 = zd.clone()
            calls.append((first, ops.distill_loss_grad(z3, vd, xd, first, gl.cuda(), targets=td, d_logprob=hard, temperature=T, rest=rest, out=z3)))
    for r, d in calls:
        loss, grad = r.loss.double().cpu(), d.double().cpu()
        assert d.dtype == z.dtype and d.shape == z.shape
        for i, (l, lp, w) in enumerate(want):
            got = float(loss[i])
            if l > 2.0 ** 128:                      # of logits 3.4e38 apart: T^2 times that is nearest to an fp32 infinity
                l = math.inf
            if not math.isfinite(l):
                assert got == l or (math.isnan(l) and math.isnan(got)), (i, got, l)
            else:
                assert abs(got - l) <= 2 * ATOL * T * T + 2 ** -22 * abs(l), (i, got, l)
            if t is not None:
                got = float(r.logprob[i])
                assert (math.isnan(lp) and math.isnan(got)) or got == lp or abs(got - lp) <= ATOL + 2 ** -22 * abs(lp), (i, got, lp)
            assert torch.equal(torch.isnan(grad[i]), torch.isnan(w)), i
            if bool(torch.isnan(w).any()):
                continue
            room = GTOL * (T * abs(float(gl[i])) + (abs(float(gh[i])) if t is not None else 0.0)) + (2.0 ** -8 * w.abs() if z.dtype == BF16 else 0.0)
            assert bool(((grad[i] - w).abs() <= room).all()), (i, float((grad[i] - w).abs().max()))
    if t is None:
        assert first.logprob is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,k,T", [(1, 1, 1, 1.0), (3, 2, 1, 2.0), (5, 7, 7, 1.0), (2, 64, 64, 0.5), (4, 255, 17, 1.0), (3, 1000, 256, 4.0), (2, 4099, 32, 1.0),
                                            (1, 32003, 5, 2.0), (600, 130, 9, 1.0), (520, 2500, 33, 3.0)])
def test_formulas(rows, vocab, k, T, rest, dtype):
    z = logits(rows * vocab, rows, vocab, dtype)
    value, index = lists(vocab + k, rows, vocab, k, rest)
    t = torch.randint(-1, vocab, (rows,), generator=torch.Generator().manual_seed(k), dtype=torch.int32)
    if rows > 2:
        t[1] = vocab                            # outside: none
        t[2] = max(0, int(index[2, 0]))         # a target that is listed, mostly
    check(z, value, index, t, T, rest)
    check(z, value, index, None, T, rest, in_place=False)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,dtype", [(2, 70001, F32), (1, 140003, BF16), (513, 20011, BF16), (512, 33001, BF16), (512, 70001, BF16), (512, 40001, F32)])
def test_long_rows(rows, vocab, dtype, rest):
    """Rows in parts, and each size of workgroup; few rows of the many are looked at."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 2.5).to(dtype)
    value, index = lists(rows, rows, vocab, 20, rest)
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(rows), dtype=torch.int32)
    gl, gh = torch.rand(rows), torch.rand(rows)
    r, d = _ops().distill_loss_with_grad(z, value.cuda(), index.cuda(), gl.cuda(), targets=t.cuda(), d_logprob=gh.cuda(), temperature=2.0, rest=rest)
    later = _ops().distill_loss_grad(z, value.cuda(), index.cuda(), r, gl.cuda(), targets=t.cuda(), d_logprob=gh.cuda(), temperature=2.0, rest=rest)
    for i in sorted({0, rows // 2, rows - 1}):
        l, lp, w = want_row(z[i].cpu().double(), value[i], index[i], int(t[i]), 2.0, rest, float(gl[i]), float(gh[i]))
        assert abs(float(r.loss[i]) - l) <= 2 * ATOL * 4 + 2 ** -22 * abs(l)
        assert abs(float(r.logprob[i]) - lp) <= ATOL + 2 ** -22 * abs(lp)
        for grad in (d, later):
            room = GTOL * 3 + (2.0 ** -8 * w.abs() if dtype == BF16 else 0.0)
            assert bool(((grad[i].cpu().double() - w).abs() <= room).all())


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,dtype", [(2048, 66001, F32), (2048, 140003, BF16), (31, 20011, F32)])
def test_gradient_on_the_logits_of_many_rows_in_parts(rows, vocab, dtype, rest):
    """Workgroups that write a row's gradient late need what others wrote over early: lists in all parts, or in the first one alone."""
    g = torch.Generator(device="cuda").manual_seed(rows + rest)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 2.0).to(dtype)
    index = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda", dtype=torch.int32)
    index[::2] %= 4000
    value = torch.log_softmax(torch.randn(rows, 25, generator=g, device="cuda"), 1)[:, :24].contiguous()
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    t[::3] %= 4000
    gl, gh = torch.rand(rows, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    apart, d = _ops().distill_loss_with_grad(z, value, index, gl, targets=t, d_logprob=gh, temperature=1.5, rest=rest)
    on = _ops().distill_loss_with_grad(z, value, index, gl, targets=t, d_logprob=gh, temperature=1.5, rest=rest, out=z)
    assert torch.equal(apart.loss, on[0].loss) and torch.equal(apart.logprob, on[0].logprob) and torch.equal(apart.stats, on[0].stats)
    assert on[1] is z and torch.equal(d, z)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(9, 300), (530, 600)])
def test_masks_and_empty_lists(rows, vocab, rest, dtype):
    z = logits(3, rows, vocab, dtype, masked=0.3)
    value, index = lists(4, rows, vocab, 12, rest)
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    z[0] = -math.inf                                       # nothing is allowed
    z[1] = -math.inf
    index[1] = -1                                          # and there is no list either
    index[2] = -1                                          # no list
    value[3] = -math.inf                                   # a list of what cannot occur
    z[4] = torch.finfo(dtype).min                          # a mask of the lowest value leaves nothing else
    z[5] = torch.finfo(dtype).min
    z[5, 7] = 1.0
    index[6, 0], value[6, 0] = 11, -math.inf
    keep = [int(i) for i in index[7] if i >= 0]            # the student allows nothing outside the list
    z[7] = -math.inf
    z[7, keep] = torch.randn(len(keep)).to(dtype)
    z[8, keep] = 0.5
    check(z, value, index, t, 1.0, rest)
    check(z, value, index, t, 3.0, rest, separate=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [False, True])
def test_nothing_finite_spreads_beyond_its_row(rest, dtype):
    z = logits(8, 7, 500, dtype)
    value, index = lists(9, 7, 500, 8, rest, missing=0.0)
    z[1, 100] = math.nan
    z[2, 499] = math.inf
    z[3, int(index[3, 2])] = math.nan                      # a listed one
    z[4, int(index[4, 0])] = math.inf
    value[5, 1] = math.nan
    value[6, 3] = math.inf
    t = torch.full((7,), 3, dtype=torch.int32)
    check(z, value, index, t, 1.0, rest)
    check(z, value, index, t, 2.0, rest, separate=False)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows", [3, 600])
def test_a_token_listed_twice(rows, rest):
    z = logits(10, rows, 77, F32)
    value, index = lists(11, rows, 77, 10, rest)
    index[:, 4] = index[:, 1]
    index[0] = 5
    t = index[:, 1].clone()
    check(z, value, index, t, 2.0, rest)


@pytest.mark.parametrize("rows", [2, 600])
def test_a_student_that_is_sure_of_its_list(rows):
    """The rest of the student is far below what one minus its list could hold, or an exponential against its best."""
    z = torch.full((rows, 400), -150.0)
    z += torch.randn(400, generator=torch.Generator().manual_seed(2))
    z[:, 17] = 3.0
    index = torch.tensor([[17, 20]], dtype=torch.int32).repeat(rows, 1)
    value = torch.log(torch.tensor([[0.6, 0.3]])).repeat(rows, 1)
    r, d = _ops().distill_loss_with_grad(z.cuda(), value.cuda(), index.cuda(), torch.ones(rows, device="cuda"), rest=True)
    l, _, w = want_row(z[0].double(), value[0], index[0], -1, 1.0, True, 1.0, 0.0)
    assert l > 10.0 and abs(float(r.loss[0]) - l) <= 2e-6 * l
    assert float(w[30]) < -1e-5 and bool(((d[0].cpu().double() - w).abs() <= GTOL).all()) and abs(float(d[0, 30]) / float(w[30]) - 1) < 1e-4


def test_gradient_against_differences():
    z = logits(20, 1, 9, F32, spread=1.0)
    value, index = lists(21, 1, 9, 4, True, missing=0.0)
    t = torch.tensor([2], dtype=torch.int32)
    for rest in (False, True):
        _, d = _ops().distill_loss_with_grad(z.cuda(), value.cuda(), index.cuda(), torch.tensor([0.7]).cuda(), targets=t.cuda(), d_logprob=torch.tensor([-0.4]).cuda(),
                                             temperature=1.5, rest=rest)

        def f(zz):
            l, lp, _ = want_row(zz, value[0], index[0], 2, 1.5, rest, 0.0, 0.0)
            return 0.7 * l - 0.4 * lp
        for j in range(9):
            step = torch.zeros(9, dtype=torch.float64)
            step[j] = 1e-5
            slope = (f(z[0].double() + step) - f(z[0].double() - step)) / 2e-5       # error: third derivative h^2, and 1e-15 / h
            assert abs(float(d[0, j]) - slope) <= 1e-6 + GTOL


def test_strides_shapes_and_streams():
    """A padded view as input and output, three axes, another stream than the current one before."""
    ops = _ops()
    big = logits(30, 6, 1100, BF16).cuda()
    z = big[:, 37:1037]
    value, index = (x.cuda() for x in lists(31, 6, 1000, 16, True))
    gl = torch.rand(6).cuda()
    out = torch.full((6, 1200), 7.0, dtype=BF16, device="cuda")
    r, d = ops.distill_loss_with_grad(z, value, index, gl, rest=True, out=out[:, 100:1100])
    r1, d1 = ops.distill_loss_with_grad(z.contiguous(), value, index, gl, rest=True)
    assert torch.equal(r.loss, r1.loss) and torch.equal(out[:, 100:1100], d1) and bool((out[:, :100] == 7).all()) and bool((out[:, 1100:] == 7).all())
    r3, d3 = ops.distill_loss_with_grad(z.contiguous().view(2, 3, 1000), value.view(2, 3, 16), index.view(2, 3, 16), gl.view(2, 3), rest=True)
    assert r3.loss.shape == (2, 3) and torch.equal(r3.loss.view(-1), r1.loss) and torch.equal(d3.view(6, 1000), d1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r4, d4 = ops.distill_loss_with_grad(z, value, index, gl, rest=True)
    side.synchronize()
    assert torch.equal(r4.loss, r1.loss) and torch.equal(d4, d1)
    empty = ops.distill_loss(z[:0], value[:0], index[:0])
    assert empty.loss.shape == (0,)


@pytest.mark.parametrize("rows,vocab", [(3, 9000), (600, 800)])
def test_captured(rows, vocab):
    ops = _ops()
    z = logits(40, rows, vocab, BF16).cuda()
    value, index = (x.cuda() for x in lists(41, rows, vocab, 16, True))
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    gl, gh = torch.rand(rows).cuda(), torch.rand(rows).cuda()

    def call():
        return ops.distill_loss_with_grad(z, value, index, gl, targets=t, d_logprob=gh, temperature=2.0, rest=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, d = call()
    for seed in (50, 51, 52):
        z.copy_(logits(seed, rows, vocab, BF16))
        graph.replay()
        torch.cuda.synchronize()
        want, wd = call()
        assert torch.equal(r.loss, want.loss) and torch.equal(d, wd) and torch.equal(r.logprob, want.logprob)


def test_refusals():
    ops = _ops()
    z = logits(60, 4, 50, F32).cuda()
    value, index = (x.cuda() for x in lists(61, 4, 50, 3, False))
    g = torch.ones(4, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    good = ops.distill_loss(z, value, index)
    for call in (lambda: ops.distill_loss(z, value[:3], index), lambda: ops.distill_loss(z, value, index[:, :2]), lambda: ops.distill_loss(z, value.double(), index),
                 lambda: ops.distill_loss(z, value, index.long()), lambda: ops.distill_loss(z.half(), value, index), lambda: ops.distill_loss(z, value[:, :0], index[:, :0]),
                 lambda: ops.distill_loss(z, value, index, temperature=0.0), lambda: ops.distill_loss(z, value, index, temperature=math.nan),
                 lambda: ops.distill_loss(z, value, index, targets=t.long()), lambda: ops.distill_loss(z, value.cpu(), index),
                 lambda: ops.distill_loss(z.t(), value, index), lambda: ops.distill_loss(z[:1].expand(4, 50), value, index),
                 lambda: ops.distill_loss(z, value.repeat(1, 100), index.repeat(1, 100)),
                 lambda: ops.distill_loss_with_grad(z, value, index, g[:3]), lambda: ops.distill_loss_with_grad(z, value, index, g, d_logprob=g),
                 lambda: ops.distill_loss_with_grad(z, value, index, g, out=torch.empty(4, 51, device="cuda")),
                 lambda: ops.distill_loss_with_grad(z, value, index, g, out=z.bfloat16()),
                 lambda: ops.distill_loss_grad(z, value, index, good, g, targets=t), lambda: ops.distill_loss_grad(z, value, index, good._replace(stats=good.stats[:2]), g)):
        with pytest.raises(B.OlsError):
            call()
