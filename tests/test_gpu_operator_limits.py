"""The operators at the ends of the sizes that they accept, against plain torch operations.

Tolerances as of the operators' own tests: 4e-6 and 2^-22 of the value for log probabilities (their sums are of positive terms, in short
partial sums)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


# 256 parts a row, each with its 32 best
@pytest.mark.parametrize("rows,vocab,dtype", [(1, 600_011, F32), (2, 600_011, F32), (1, 1_100_003, BF16), (1, 1 << 24, F32)])
def test_most_alternatives_of_the_longest_rows(rows, vocab, dtype):
    z = torch.randn(rows, vocab, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").to(dtype)
    r = _ops().token_logprobs(z, None, top=32)
    d = z.double()
    lse = torch.logsumexp(d, 1)
    v, i = torch.sort(d, dim=1, descending=True, stable=True)
    assert torch.equal(r.top_index, i[:, :32].to(torch.int32))
    want = v[:, :32] - lse[:, None]
    assert ((r.top_logprob.double() - want).abs() <= 4e-6 + 2.0 ** -22 * want.abs()).all()
    assert ((r.logsumexp.double() - lse).abs() <= 4e-6 + 2.0 ** -22 * lse.abs()).all()


@pytest.mark.parametrize("vocab", [70_001, 600_011])
def test_ties_across_all_parts(vocab):
    """What is equal everywhere, equal from some part on, and equal but for a few."""
    z = torch.zeros(4, vocab, device="cuda")
    z[1, vocab // 2:] = 1.0
    z[2, 5::997] = 2.0
    z[3, vocab - 3:] = 3.0
    best = _ops().token_logprobs(z[:2], None, top=32).top_index.tolist() + _ops().token_logprobs(z[2:], None, top=32).top_index.tolist()
    assert best[0] == list(range(32)) and best[1] == list(range(vocab // 2, vocab // 2 + 32))
    assert best[2] == list(range(5, 5 + 32 * 997, 997)) and best[3] == [vocab - 3, vocab - 2, vocab - 1, *range(29)]
    one = torch.full((1, vocab), -math.inf, device="cuda")
    one[0, vocab - 7] = 0.5
    assert _ops().token_logprobs(one, None, top=32).top_index.tolist() == [[vocab - 7] + [-1] * 31]


def _device_us(call):
    """Of the least of five runs of ten calls."""
    call()
    times = []
    for _ in range(5):
        a, b = torch.cuda.Event(True), torch.cuda.Event(True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(10):
            call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 100)
    return min(times)


def test_rows_of_one_value_take_little_longer_than_others():
    """What ties is not compared pair by pair: 65 us beside 45, and 23 ms where all that the parts hold was."""
    random, equal = torch.randn(1, 600_011, device="cuda"), torch.zeros(1, 600_011, device="cuda")
    assert _device_us(lambda: _ops().token_logprobs(equal, None, top=32)) <= 8 * _device_us(lambda: _ops().token_logprobs(random, None, top=32))


@pytest.mark.parametrize("rows", [1 << 21, (1 << 21) + 3, (1 << 24) + 5])
def test_rows_of_logits_beyond_a_launch(rows):
    """A launch has fewer than 2^32 threads, 256 of them for a row."""
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(rows, 9, generator=g, device="cuda").to(BF16)
    t = torch.randint(-1, 9, (rows,), generator=g, device="cuda", dtype=torch.int32)
    up, h = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    r, d = _ops().token_logprobs_with_grad(z, t, up, h, top=2)
    later = _ops().token_logprobs_grad(z, t, r, up, h)
    for pick in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice((1 << 21) - 500, (1 << 21) + 500), slice(rows - 1000, rows)):
        logp = torch.log_softmax(z[pick].double(), 1)
        real = t[pick] >= 0
        want = torch.where(real, logp.gather(1, t[pick].long().clamp(min=0)[:, None])[:, 0], 0.0)
        p, s = logp.exp(), -(logp.exp() * logp).sum(1, keepdim=True)
        hot = torch.zeros_like(p).scatter_(1, t[pick].long().clamp(min=0)[:, None], 1.0)
        grad = torch.where(real, up[pick], 0.0).double()[:, None] * (hot - p) - h[pick].double()[:, None] * p * (logp + s)
        v, i = torch.sort(z[pick], dim=1, descending=True, stable=True)
        assert ((r.logprob[pick].double() - want).abs() <= 4e-6 + 2.0 ** -22 * want.abs()).all()
        assert ((r.entropy[pick].double() - s[:, 0]).abs() <= 4e-6).all()
        assert torch.equal(r.top_index[pick], i[:, :2].to(torch.int32))
        for got in (d, later):
            assert ((got[pick].double() - grad).abs() <= 2e-5 + 2.0 ** -8 * grad.abs()).all()


def test_lookup_beyond_a_launch():
    """2^24 ids of rows that take a workgroup each: 34 GB of results."""
    n, width = 1 << 24, 1025
    g = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randn(7, width, generator=g, device="cuda").to(BF16)
    ids = torch.randint(-1, 7, (n,), generator=g, device="cuda", dtype=torch.int32)
    out = torch.full((n, width), 9.0, dtype=BF16, device="cuda")
    _ops().embed(table, ids, 1.0, out=out)
    rows = torch.cat([table, torch.zeros(1, width, dtype=BF16, device="cuda")])     # -1: the last
    for first in range(0, n, 1 << 20):
        part = slice(first, first + (1 << 20))
        assert torch.equal(out[part], rows[ids[part].long()]), first
    del out
    torch.cuda.empty_cache()


def test_gradients_of_no_rows_beyond_a_launch():
    """A weight's gradient of more than 2^32 elements is cleared whole: 8.6 GB."""
    from paper_2002_09539_amd import binding as B
    width, hidden = 65_537, 65_536
    g = torch.ones(width, hidden, dtype=BF16, device="cuda")
    f = B.ols_ffn()
    f.groups, f.act, f.dtype, f.weight_dtype, f.grad_dtype = 1, B.OLS_ACT_SILU, B.OLS_BF16, B.OLS_BF16, B.OLS_BF16
    f.rows, f.width, f.hidden, f.out = 0, width, hidden, 1
    f.g_gate = B.ols_matrix(g.data_ptr(), hidden, 0)
    B.ols_gated_ffn_grad(f, torch.cuda.current_stream().cuda_stream)
    assert all(int(torch.count_nonzero(g[i: i + 4096])) == 0 for i in range(0, width, 4096))
    del g
    torch.cuda.empty_cache()


def test_inputs_laid_out_beyond_a_launch():
    """More than 2^32 units of eight elements: 69 GB of rows that do not lie on 16 bytes, and as much to lay them out."""
    rows, width, hidden, out = 1 << 24, 2049, 8, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).to(BF16)  # noqa: E731
    wg, wu, wd = r(width, hidden, std=width ** -0.5), r(width, hidden, std=width ** -0.5), r(hidden, out, std=hidden ** -0.5)
    x = torch.empty(rows, width, dtype=BF16, device="cuda")
    for i in range(0, rows, 1 << 20):
        x[i: i + (1 << 20)] = r(1, width, std=1.0)             # of every 2^20 rows all alike: results as well
    y = _ops().gated_ffn(x, wg, wu, wd, "relu")
    for i in range(0, rows, 1 << 20):
        part = y[i: i + (1 << 20)]
        a, b = x[i].double() @ wg.double(), x[i].double() @ wu.double()
        want = (a.clamp(min=0) * b) @ wd.double()
        assert torch.equal(part, part[:1].expand_as(part)), i
        assert float((part[0].double() - want).norm()) <= 1e-2 * float(want.norm()), i
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("apart", [False, True])
def test_gradient_tables_beyond_a_launch(apart):
    """137 GB of rows to clear, side by side and a little apart: more pieces of 64 KiB (of one row each) than a launch numbers."""
    vocab, width = (1 << 22) + 100, 16_385
    whole = torch.empty(vocab, width + apart, dtype=BF16, device="cuda").fill_(1.0)
    out = whole[:, :width]
    ids = torch.tensor([vocab - 1, 5, 5], dtype=torch.int32, device="cuda")
    _ops().embed_grad(ids, torch.ones(3, width, dtype=BF16, device="cuda"), vocab, out=out)
    assert (out[5] == 2).all() and (out[vocab - 1] == 1).all()
    out[5], out[vocab - 1] = 0.0, 0.0
    step = 1 << 18
    assert all(int(torch.count_nonzero(out[i: i + step])) == 0 for i in range(0, vocab, step))
    assert not apart or (whole[:, width] == 1).all()
    del out, whole
    torch.cuda.empty_cache()
