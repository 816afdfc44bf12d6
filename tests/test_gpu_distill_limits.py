"""Distillation, quantisers and the moving of states with more rows than one launch takes, and without a gradient of the loss, against plain torch
operations.

Tolerances as in the operators' own tests: a loss at temperature 1 within 8e-6 and 2^-22 of itself, log probabilities 4e-6 and 2^-22, gradients 2e-5
of their factors and, in bf16, 2^-8 of themselves; quantised values and scales are equal."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
LAUNCH = 1 << 21                    # rows of few logits, or of all workers to be quantised


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _distill_want(z, value, index, t, gl, gh):
    """Loss, log probability and gradient of rows whose lists name two tokens, at temperature 1, the rest left out."""
    logp = torch.log_softmax(z.double(), 1)
    p, at = logp.exp(), index.long()
    q = torch.softmax(value.double(), 1)
    loss = (q * (q.log() - logp.gather(1, at))).sum(1)
    grad = gl.double()[:, None] * p.scatter_add(1, at, -q)
    real = (t >= 0)[:, None]
    place = t.long().clamp(min=0)[:, None]
    lp = torch.where(real, logp.gather(1, place), 0.0)[:, 0]
    hot = torch.zeros_like(p).scatter_(1, place, 1.0)
    return loss, lp, grad + torch.where(real, gh.double()[:, None] * (hot - p), 0.0)


def test_distillation_of_rows_beyond_a_launch():
    ops, rows, vocab = _ops(), LAUNCH + 3, 10
    g = torch.Generator(device="cuda").manual_seed(1)
    z = (torch.randn(rows, vocab, generator=g, device="cuda") * 2).to(BF16)
    index = torch.randint(0, 5, (rows, 2), generator=g, device="cuda", dtype=torch.int32)
    index[:, 1] += 5
    value = torch.randn(rows, 2, generator=g, device="cuda")
    t = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    gl, gh = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    alone = ops.distill_loss(z, value, index, targets=t)
    r, d = ops.distill_loss_with_grad(z, value, index, gl, targets=t, d_logprob=gh)
    later = ops.distill_loss_grad(z, value, index, alone, gl, targets=t, d_logprob=gh)
    on = z.clone()
    ops.distill_loss_with_grad(on, value, index, gl, targets=t, d_logprob=gh, out=on)
    assert torch.equal(on, d) and torch.equal(alone.stats, r.stats)
    for pick in (slice(0, 1000), slice(rows // 2, rows // 2 + 1000), slice(LAUNCH - 500, rows)):
        loss, lp, grad = _distill_want(z[pick], value[pick], index[pick], t[pick], gl[pick], gh[pick])
        room = 2e-5 * (gl[pick].abs() + gh[pick].abs()).double()[:, None] + 2.0 ** -8 * grad.abs()
        for got in (alone, r):
            assert bool(((got.loss[pick].double() - loss).abs() <= 8e-6 + 2.0 ** -22 * loss.abs()).all())
            assert bool(((got.logprob[pick].double() - lp).abs() <= 4e-6 + 2.0 ** -22 * lp.abs()).all())
        for got in (d, later):
            assert bool(((got[pick].double() - grad).abs() <= room).all())


@pytest.mark.parametrize("rows,vocab", [(5, 40), (3, 30011), (700, 2500)])
def test_no_gradient_of_the_loss(rows, vocab):
    """d_loss None: that of the log probabilities alone, as token_logprobs_with_grad computes it; without either, zeros."""
    ops = _ops()
    g = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.randn(rows, vocab, generator=g, device="cuda")
    best = ops.token_logprobs(z + 0.5 * torch.randn(rows, vocab, generator=g, device="cuda"), None, top=8)
    t = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    gh = torch.randn(rows, generator=g, device="cuda")
    _, want = ops.token_logprobs_with_grad(z, t, gh)
    for rest in (False, True):
        r, d = ops.distill_loss_with_grad(z, best.top_logprob, best.top_index, None, targets=t, d_logprob=gh, temperature=2.0, rest=rest)
        later = ops.distill_loss_grad(z, best.top_logprob, best.top_index, r, None, targets=t, d_logprob=gh, temperature=2.0, rest=rest)
        for got in (d, later):
            assert bool(((got - want).abs() <= 2 * 2e-5 * gh.abs()[:, None]).all())
        _, none = ops.distill_loss_with_grad(z, best.top_logprob, best.top_index, None, temperature=2.0, rest=rest)
        assert bool((none == 0).all())


@pytest.mark.parametrize("m,rows", [(1, LAUNCH + 3), (3, LAUNCH // 3 + 5), (2, LAUNCH + 7)])
def test_quantised_rows_beyond_a_launch(m, rows):
    """A launch's rows end inside every worker's."""
    x = torch.randn(m, rows, 8, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda")
    r = _ops().quantize_rows(x)
    scale = (x.abs().amax(2).double() / 127).float()
    assert torch.equal(r.scale, scale)
    for i in range(m):                                      # in 64 bits, a worker at a time
        assert torch.equal(r.q[i], torch.round(x[i].double() / scale[i].double()[:, None]).to(torch.int8))


def test_states_of_requests_beyond_a_launch():
    """65 535 requests of sixty tensors, five pieces of 4096 bytes each: 64 GB, of which a launch takes 55 924 requests."""
    ops, batch, size, n = _ops(), 65_535, 16_385, 60
    src = torch.randint(0, 256, (n, 1, 2, size), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda", dtype=torch.uint8)
    parent = torch.randint(0, 2, (batch, 1), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda", dtype=torch.int32)
    out = torch.empty(n, batch, 1, size, device="cuda", dtype=torch.uint8)
    ops.beam_reorder([s.expand(batch, 2, size) for s in src], parent, out=list(out))
    cut = ((1 << 24) - 1) // (5 * n)
    assert cut < batch
    for pick in (slice(0, 200), slice(cut - 200, cut + 200), slice(batch - 200, batch)):
        for i in range(n):
            assert torch.equal(out[i, pick, 0], src[i, 0][parent[pick, 0].long()]), (i, pick)
    del out
    torch.cuda.empty_cache()
