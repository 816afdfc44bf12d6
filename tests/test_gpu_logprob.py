"""Log probabilities of given tokens with entropy and best alternatives, and their gradient, against 64 bits.

Tolerances.  In fp32 the sums s and t have relative errors of a few 2^-24 (sums of positive terms in short partial sums,
each exponential good to 2 units in the last place plus 2^-24 |z - m| from rounding its argument); logarithm, logsumexp and
logprob then carry absolute errors of that size plus half a unit in their own last place.  ATOL = 4e-6 holds ten times that
for |z - m| <= 60.  Entropy is a difference of log s and t / s, both below 17: the same absolute bound.  A gradient
entry is a product of p (relative 1e-5) with upstream gradients of order one: 2e-5 absolute, plus the storage rounding."""
import math

import numpy as np
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ATOL, GTOL = 4e-6, 2e-5


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _logits(seed, rows, vocab, dtype, masked=0.0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * spread
    if masked:
        z[torch.rand(rows, vocab, generator=g) < masked] = -math.inf
    return z.to(dtype)


def _want(z, t, g_lp=None, g_h=None, top=0):
    z = z.double()
    rows, vocab = z.shape
    out = {k: [] for k in ("logprob", "entropy", "logsumexp", "top_logprob", "top_index", "grad")}
    for i in range(rows):
        row = z[i]
        bad = bool(torch.isnan(row).any() or (row == math.inf).any())
        empty = bool((row == -math.inf).all())
        has = t is not None and 0 <= int(t[i]) < vocab
        if bad or empty:
            fill = math.nan if bad else -math.inf
            out["logsumexp"].append(fill)
            out["entropy"].append(math.nan if bad else 0.0)
            out["logprob"].append(fill if has else 0.0)
            if bad and has is False:
                out["logprob"][-1] = 0.0
            out["top_logprob"].append([fill] * top)
            out["top_index"].append([-1] * top)
            out["grad"].append(torch.full((vocab,), math.nan if bad else 0.0, dtype=torch.float64))
            continue
        lse = torch.logsumexp(row, 0)
        row0 = row - row.max()            # at the lowest value, log of the vocabulary is below a 64-bit number's last place
        logp = row0 - torch.logsumexp(row0, 0)
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
        h = -plogp.sum()
        out["logsumexp"].append(float(lse))
        out["entropy"].append(float(h))
        out["logprob"].append(float(logp[int(t[i])]) if has else 0.0)
        order = torch.argsort(-row, stable=True)[:top]
        out["top_index"].append([int(j) if row[j] > -math.inf else -1 for j in order])
        out["top_logprob"].append([float(logp[j]) if row[j] > -math.inf else -math.inf for j in order])
        if g_lp is not None:
            hot = torch.zeros(vocab, dtype=torch.float64)
            if has:
                hot[int(t[i])] = 1.0
            a, b = (float(g_lp[i]) if has else 0.0), float(g_h[i])
            out["grad"].append(a * (hot - p) - b * (plogp + p * h))
    return {k: (torch.stack(v) if k == "grad" and v else np.array(v)) for k, v in out.items()}


def _close(got, want, tol):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    room = tol + 2.0 ** -22 * np.abs(want[fine])
    assert (np.abs(got[fine] - want[fine]) <= room).all(), np.abs(got[fine] - want[fine]).max()


def _check(z, t, top, with_grad=True):
    zd, td = z.cuda(), None if t is None else t.cuda()
    rows, vocab = z.shape
    g = torch.Generator().manual_seed(rows)
    g_lp, g_h = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    want = _want(z, t, g_lp, g_h, top)
    r = _ops().token_logprobs(zd, td, top=top)
    results = [r]
    if with_grad:
        fused, d = _ops().token_logprobs_with_grad(zd, td, g_lp.cuda(), g_h.cuda(), top=top)
        later = _ops().token_logprobs_grad(zd, td, r, g_lp.cuda(), g_h.cuda())
        results.append(fused)
        for grad in (d, later):
            assert grad.dtype == z.dtype
            w = want["grad"].numpy()
            got = grad.double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(w))
            fine = ~np.isnan(w)
            room = GTOL + (2.0 ** -8 * np.abs(w[fine]) if z.dtype == BF16 else 0.0)
            assert (np.abs(got[fine] - w[fine]) <= room).all(), np.abs(got[fine] - w[fine]).max()
    for q in results:
        _close(q.logprob, want["logprob"], ATOL)
        _close(q.entropy, want["entropy"], ATOL)
        _close(q.logsumexp, want["logsumexp"], ATOL)
        if top:
            assert np.array_equal(q.top_index.cpu().numpy(), want["top_index"])
            _close(q.top_logprob, want["top_logprob"], ATOL)


def _targets(seed, rows, vocab):
    r = np.random.RandomState(seed)
    t = r.randint(0, vocab, rows)
    t[r.uniform(size=rows) < 0.15] = -1
    t[r.uniform(size=rows) < 0.1] = vocab
    return torch.tensor(t, dtype=torch.int32)


# one token; less than a vector; odd rows; one workgroup's registers and one more; parts of few rows; more than the largest workgroup
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 257, 32), (600, 129, 5), (2, 4096, 8), (3, 4097, 8), (530, 8193, 4),
                                            (520, 33001, 2), (2, 70001, 20), (1, 140003, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("masked", [0.0, 0.5])
def test_rows(rows, vocab, top, dtype, masked):
    z = _logits(rows * 7 + vocab, rows, vocab, dtype, masked)
    keep = min(rows, 40)                     # the reference walks row by row: the last rows stand for the others
    t = _targets(vocab, rows, vocab)
    if keep == rows:
        _check(z, t, top)
        return
    r = _ops().token_logprobs(z.cuda(), t.cuda(), top=top)
    want = _want(z[-keep:], t[-keep:], None, None, top)
    _close(r.logprob[-keep:], want["logprob"], ATOL)
    _close(r.entropy[-keep:], want["entropy"], ATOL)
    assert np.array_equal(r.top_index[-keep:].cpu().numpy(), want["top_index"])


@pytest.mark.parametrize("rows,vocab", [(515, 257), (513, 8193), (512, 33001), (514, 66000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_of_many_rows(rows, vocab, dtype):
    """Rows that fill the device: a workgroup holds each, and the gradient comes from its registers."""
    z, t = _logits(vocab, rows, vocab, dtype, 0.1), _targets(vocab, rows, vocab)
    g = torch.Generator().manual_seed(1)
    g_lp, g_h = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    zd = z.cuda()
    r, d = _ops().token_logprobs_with_grad(zd, t.cuda(), g_lp.cuda(), g_h.cuda())
    pick = [0, 1, rows // 2, rows - 1]
    want = _want(z[pick], t[pick], g_lp[pick], g_h[pick])
    got = d[pick].double().cpu()
    room = GTOL + (2.0 ** -8 * want["grad"].abs() if dtype == BF16 else 0.0)
    assert ((got - want["grad"]).abs() <= room).all()
    _close(r.logprob[pick], want["logprob"], ATOL)
    same, place = _ops().token_logprobs_with_grad(zd, t.cuda(), g_lp.cuda(), g_h.cuda(), out=zd)     # over the logits
    assert place is zd and torch.equal(zd, d) and torch.equal(same.logprob, r.logprob)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [5, 3000, 40000])
def test_masks_and_what_is_no_number(dtype, vocab):
    low = float(torch.finfo(dtype).min)
    high = float(torch.finfo(dtype).max)
    z = _logits(2, 10, vocab, dtype)
    z[0] = -math.inf                          # nothing can occur
    z[1] = low                                # everything equally
    z[2, 1:] = low                            # masked by the lowest value
    z[3] = -math.inf
    z[3, vocab // 2] = 1.0                    # one token
    z[4, 3] = math.nan
    z[5, 4] = math.inf
    z[6, 2:] = -math.inf
    z[7, 1] = high                            # differences that overflow
    z[7, 2] = low
    z[8] = math.nan
    z[9, :3] = 0.0
    z[9, 0] = -0.0
    t = torch.tensor([0, 1, 0, vocab // 2, 3, 1, vocab - 1, 1, 0, -5], dtype=torch.int32)
    _check(z, t, min(vocab, 4))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(2, 100), (2, 9000), (600, 2050)])
def test_ties_go_to_the_lowest_index(dtype, rows, vocab):
    z = torch.zeros(rows, vocab)
    z[0, vocab // 3:] = 1.0
    z[1] = torch.arange(vocab) % 3
    r = _ops().token_logprobs(z.to(dtype).cuda(), None, top=32)
    assert r.top_index[0].tolist() == list(range(vocab // 3, vocab // 3 + 32))
    assert r.top_index[1].tolist() == list(range(2, 2 + 3 * 32, 3))
    assert rows < 3 or r.top_index[2].tolist() == list(range(32))


def test_sorted_rows():
    """All of the best in one lane's vectors, or in one wavefront's."""
    for vocab in (2000, 50000):
        z = torch.stack([-torch.arange(vocab), torch.arange(vocab)]).float() * 1e-3
        r = _ops().token_logprobs(z.cuda(), None, top=20)
        assert r.top_index[0].tolist() == list(range(20)) and r.top_index[1].tolist() == list(range(vocab - 1, vocab - 21, -1))


def test_strided_rows_and_axes():
    z = torch.randn(6, 5, 50, device="cuda")
    t = torch.randint(0, 50, (6, 5), device="cuda", dtype=torch.int32)
    r = _ops().token_logprobs(z, t, top=3)
    assert r.logprob.shape == (6, 5) and r.top_index.shape == (6, 5, 3)
    wide = torch.randn(7, 61, device="cuda").to(BF16)
    part = wide[:, 3:54]
    _close(_ops().token_logprobs(part).logsumexp, _want(part.cpu(), None)["logsumexp"], ATOL)
    before = wide.clone()
    g = torch.ones(7, device="cuda")
    _, d = _ops().token_logprobs_with_grad(part, torch.zeros(7, dtype=torch.int32, device="cuda"), g, out=part)
    assert torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 54:], before[:, 54:]) and not torch.equal(wide, before)
    assert _ops().token_logprobs(torch.zeros(0, 9, device="cuda")).logprob.shape == (0,)


def test_gradient_against_differences():
    """Central differences in 64 bits of what the definition gives; step 1e-4, whose error is of order 1e-8."""
    z, t = _logits(5, 3, 9, F32).double(), torch.tensor([2, 8, 0])
    g_lp, g_h = torch.tensor([0.7, -1.1, 0.3]), torch.tensor([-0.4, 0.9, 1.3])

    def value(z):
        logp = torch.log_softmax(z, 1)
        return (g_lp * logp[torch.arange(3), t] - g_h * (logp.exp() * logp).sum(1)).sum()

    _, d = _ops().token_logprobs_with_grad(z.float().cuda(), t.int().cuda(), g_lp.cuda(), g_h.cuda())
    for i in range(3):
        for j in range(9):
            e = torch.zeros_like(z)
            e[i, j] = 1e-4
            assert abs(float((value(z.float().double() + e) - value(z.float().double() - e)) / 2e-4) - float(d[i, j])) <= 1e-5


def test_rows_beyond_32_bit_offsets():
    rows, vocab = 18, 2 ** 27 // 16 * 16           # 18 rows of 2^23 + .. logits at a stride that passes 2^31 elements
    vocab = 1000
    stride = 2 ** 27
    big = torch.zeros((rows - 1) * stride + vocab, dtype=BF16, device="cuda")
    z = torch.as_strided(big, (rows, vocab), (stride, 1))
    fresh = torch.randn(rows, vocab, device="cuda").to(BF16)
    z.copy_(fresh)
    a, b = _ops().token_logprobs(z, top=2), _ops().token_logprobs(fresh, top=2)
    assert torch.equal(a.logsumexp, b.logsumexp) and torch.equal(a.top_index, b.top_index)


def test_in_a_graph():
    z = torch.randn(4, 9001, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _ops().token_logprobs(z, t, top=4)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = _ops().token_logprobs(z, t, top=4)
    for _ in range(3):
        z.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = _ops().token_logprobs(z, t, top=4)
        assert torch.equal(got.logprob, want.logprob) and torch.equal(got.top_index, want.top_index)


def test_refusals():
    ops = _ops()
    z, t = torch.zeros(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    g = torch.zeros(3, device="cuda")
    for call in [lambda: ops.token_logprobs(z.double()), lambda: ops.token_logprobs(z, t.long()), lambda: ops.token_logprobs(z, t[:2]),
                 lambda: ops.token_logprobs(z, t, top=9), lambda: ops.token_logprobs(z, t, top=-1), lambda: ops.token_logprobs(z.t()),
                 lambda: ops.token_logprobs(z.cpu()), lambda: ops.token_logprobs(torch.zeros(3, 64, device="cuda"), t, top=33),
                 lambda: ops.token_logprobs_with_grad(z, t, g.double()), lambda: ops.token_logprobs_with_grad(z, t, g, out=z.to(BF16)),
                 lambda: ops.token_logprobs_with_grad(z, t, g[:2])]:
        with pytest.raises(B.OlsError):
            call()
