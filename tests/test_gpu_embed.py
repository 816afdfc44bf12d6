"""Embedding lookup with scaling and its gradient by sorted tokens, against plain sums in 64 bits.

Tolerances.  The lookup is one fp32 product rounded to the result's type: half a unit in the last place of each, so 2^-24
relative (fp32), 2^-8 (bf16, with the product's own rounding).  A gradient entry is a sum of k rows in fp32, each addition
rounded by 2^-24 of the running sum: at most k 2^-24 of the sum of magnitudes (the bound used), then the product and the
storage rounding."""
import numpy as np
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = {F32: 2.0 ** -23, BF16: 2.0 ** -8}


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _tokens(seed, shape, vocab, law="words"):
    r = np.random.RandomState(seed)
    if law == "one":
        t = np.full(shape, vocab // 2)
    else:
        t = np.minimum((vocab + 1.0) ** r.uniform(size=shape), vocab).astype(np.int64) - 1
        t[r.uniform(size=shape) < 0.1] = -1
        t[r.uniform(size=shape) < 0.05] = vocab           # one past the table: no token either
        t[r.uniform(size=shape) < 0.02] = 2 ** 31 - 1
    return torch.tensor(t, dtype=torch.int32, device="cuda")


def _want_lookup(table, tokens, scale):
    t = tokens.long().cpu()
    real = (t >= 0) & (t < table.shape[0])
    return torch.where(real[..., None], table.double().cpu()[t.clamp(0, table.shape[0] - 1)] * scale, torch.zeros((), dtype=torch.float64))


@pytest.mark.parametrize("vocab,width,n", [(7, 1, 1), (50, 3, 64), (1000, 129, 300), (333, 8, 5), (513, 2056, 33), (64, 512, 0)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_lookup(vocab, width, n, dtype, out_dtype):
    g = torch.Generator(device="cuda").manual_seed(vocab + n)
    table = torch.randn(vocab, width, device="cuda", generator=g).to(dtype)
    tokens = _tokens(n, (n,), vocab)
    got = _ops().embed(table, tokens, 3.25, dtype=out_dtype)
    want = _want_lookup(table, tokens, 3.25)
    assert got.dtype == out_dtype and got.shape == (n, width)
    assert ((got.double().cpu() - want).abs() <= EPS[out_dtype] * want.abs()).all()


def test_lookup_of_workers_whose_tables_lie_in_parameter_rows():
    m, vocab, width, ld = 3, 41, 20, 1024
    x = torch.randn(m, ld, device="cuda")
    table = x[:, 12: 12 + vocab * width].unflatten(1, (vocab, width))
    tokens = _tokens(3, (m, 4, 9), vocab)
    got = _ops().embed(table, tokens)
    for w in range(m):
        assert torch.equal(got[w].double().cpu(), _want_lookup(table[w], tokens[w], 1.0))


def test_lookup_of_odd_strides_and_addresses():
    base = torch.randn(1 + 30 * 37, device="cuda").to(BF16)
    table = base[1:].unflatten(0, (30, 37))[:, :35]          # rows on odd elements, 37 apart
    tokens = _tokens(4, (200,), 30)
    assert torch.equal(_ops().embed(table, tokens, 2.0).double().cpu(), _want_lookup(table, tokens, 2.0))


def _check_grad(got, tokens, d_out, vocab, scale, before=None):
    t, d = tokens.long().cpu().reshape(-1), d_out.double().cpu().reshape(-1, d_out.shape[-1])
    real = (t >= 0) & (t < vocab)
    want = torch.zeros(vocab, d.shape[1], dtype=torch.float64)
    size = torch.zeros_like(want)
    count = torch.zeros(vocab, dtype=torch.float64)
    want.index_put_((t[real],), d[real], accumulate=True)
    size.index_put_((t[real],), d[real].abs(), accumulate=True)
    count.index_put_((t[real],), torch.ones(int(real.sum()), dtype=torch.float64), accumulate=True)
    base = torch.zeros_like(want) if before is None else before.double().cpu()
    want = base + scale * want
    room = abs(scale) * (count[:, None] + 2) * 2.0 ** -24 * size + EPS[got.dtype] * want.abs() + 2.0 ** -23 * base.abs()
    off = (got.double().cpu() - want).abs()
    assert (off <= room).all(), float((off - room).max())
    if before is not None:
        assert torch.equal(got.cpu()[count == 0], before.cpu()[count == 0])


# 4096 ids: one workgroup's; 4097: two; 20 000 with 2 ids: long runs; vocab of 511 / 512: one and two passes of 9 bits
GRADS = [(7, 1, 1, "words"), (1, 5, 64, "one"), (50, 3, 63, "words"), (511, 129, 4096, "words"), (512, 72, 4097, "words"),
         (3, 520, 20000, "words"), (300, 1032, 9000, "one"), (262144, 8, 5000, "words"), (90, 16, 0, "words")]


@pytest.mark.parametrize("vocab,width,n,law", GRADS)
@pytest.mark.parametrize("dtype,grad", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
def test_gradient(vocab, width, n, law, dtype, grad):
    tokens = _tokens(n, (n,), vocab, law)
    d_out = torch.randn(n, width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    got = _ops().embed_grad(tokens, d_out, vocab, 0.5, dtype=grad)
    assert got.dtype == grad
    _check_grad(got, tokens, d_out, vocab, 0.5)
    assert torch.equal(got, _ops().embed_grad(tokens, d_out, vocab, 0.5, dtype=grad))     # one order of every sum


@pytest.mark.parametrize("n", [100, 5000])
def test_gradient_of_workers_in_gradient_rows_and_accumulated(n):
    m, vocab, width = 3, 77, 24
    g = torch.randn(m, 4 + vocab * width + 9, device="cuda")
    before = g.clone()
    out = g[:, 4: 4 + vocab * width].unflatten(1, (vocab, width))
    tokens = _tokens(n, (m, n), vocab)
    d_out = torch.randn(m, n, width, device="cuda")
    _ops().embed_grad(tokens, d_out, vocab, 2.0, out=out, accumulate=True, workers=m)
    for w in range(m):
        _check_grad(out[w], tokens[w], d_out[w], vocab, 2.0, before=before[w, 4: 4 + vocab * width].view(vocab, width))
    assert torch.equal(g[:, :4], before[:, :4]) and torch.equal(g[:, 4 + vocab * width:], before[:, 4 + vocab * width:])
    _ops().embed_grad(tokens, d_out, vocab, 2.0, out=out, workers=m)
    for w in range(m):
        _check_grad(out[w], tokens[w], d_out[w], vocab, 2.0)


def test_gradient_is_the_lookups():
    """d/dE of sum(out * c) by differences: the lookup is linear, so a step of one is exact up to rounding."""
    vocab, width, n = 11, 5, 40
    tokens = _tokens(9, (n,), vocab)
    table, c = torch.randn(vocab, width, device="cuda"), torch.randn(n, width, device="cuda")
    grad = _ops().embed_grad(tokens, c, vocab, 1.5)
    base = (_ops().embed(table, tokens, 1.5).double() * c.double()).sum()
    for v, j in [(0, 0), (3, 4), (10, 2)]:
        moved = table.clone()
        moved[v, j] += 1.0
        diff = (_ops().embed(moved, tokens, 1.5).double() * c.double()).sum() - base
        assert abs(float(diff) - float(grad[v, j])) <= 1e-4


def test_not_a_number_stays_in_its_row():
    tokens = torch.tensor([1, 2, 1, 0], dtype=torch.int32, device="cuda")
    d = torch.ones(4, 9, device="cuda")
    d[2, 3] = float("nan")
    d[1, 0] = float("inf")
    got = _ops().embed_grad(tokens, d, 4).cpu()
    want = torch.tensor([1.0, 2.0, 1.0, 0.0])[:, None].repeat(1, 9)
    want[1, 3], want[2, 0] = float("nan"), float("inf")
    assert torch.equal(torch.nan_to_num(got, nan=-7.0), torch.nan_to_num(want, nan=-7.0))


def test_runs_on_the_current_stream_and_in_a_graph():
    ops = _ops()
    tokens = _tokens(1, (700,), 50)
    d = torch.randn(700, 40, device="cuda")
    want = ops.embed_grad(tokens, d, 50)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ops.embed_grad(tokens, d, 50)
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = ops.embed_grad(tokens, d, 50)
    for k in range(3):
        d.mul_(2.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want * 2.0 ** (k + 1))


def test_refusals():
    ops = _ops()
    table, tokens = torch.zeros(5, 4, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in [lambda: ops.embed(table, tokens.long()), lambda: ops.embed(table.half(), tokens), lambda: ops.embed(table.t(), tokens),
                 lambda: ops.embed(table.cpu(), tokens), lambda: ops.embed(table[None].repeat(2, 1, 1), tokens),
                 lambda: ops.embed(table, tokens, out=torch.zeros(3, 5, device="cuda")),
                 lambda: ops.embed_grad(tokens, torch.zeros(2, 4, device="cuda"), 5),
                 lambda: ops.embed_grad(tokens, torch.zeros(3, 4, device="cuda"), 5, accumulate=True),
                 lambda: ops.embed_grad(tokens, torch.zeros(3, 4, device="cuda"), 0),
                 lambda: ops.embed_grad(tokens, torch.zeros(3, 4, device="cuda"), 5, workers=2),
                 lambda: ops.embed_grad(tokens, torch.zeros(3, 4, device="cuda"), 5, out=torch.zeros(6, 4, device="cuda"))]:
        with pytest.raises(B.OlsError):
            call()
