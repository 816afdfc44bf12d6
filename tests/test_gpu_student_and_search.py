"""Distillation, beam search and products in 8 bits together, as the token model uses them: a student in the rows of a Session that learns
from a teacher's lists, and searches with weights as they are and in 8 bits.

Tolerances: gradients and losses as for the token model's own (fp32 3e-5 of the norm, bf16 2e-2, of the loss 1e-5 and 2e-2)."""
import math

import numpy as np
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

VOCAB, CONTEXT, WIDTH, HIDDEN = 70, 3, 12, 40


def _setup(dtype=torch.float32, m=3, batch=24):
    from paper_2002_09539_amd.session import Session
    from paper_2002_09539_amd.token_model import TokenModel, text
    model = TokenModel(VOCAB, CONTEXT, WIDTH, HIDDEN, dtype=dtype)
    teacher = TokenModel(VOCAB, CONTEXT, WIDTH, 2 * HIDDEN)
    w = np.lib.stride_tricks.sliding_window_view(text(VOCAB, m * batch + 3, 5), 4)[: m * batch].reshape(m, batch, 4).copy()
    s = Session(m, model.d, 2, 0.5, 0.2, 0.9)
    s.set_option(B.OLS_OPT_SERIALIZE, 0)
    s.init_params(model.init(3))
    params = torch.from_numpy(teacher.init(7)).cuda() * 1.5
    return model, teacher, params, s, s.upload(w[..., :3]), s.upload(w[..., 3]), w


def _logits(model, row, contexts):
    p = {n: row[model.offsets[n]: model.offsets[n] + a * b].view(a, b) for n, (a, b) in model.shapes.items()}
    x = (p["table"][contexts] * model.scale).reshape(len(contexts), -1)
    return (torch.nn.functional.silu(x @ p["w_gate"]) * (x @ p["w_up"])) @ p["w_down"]


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 3e-5), (torch.bfloat16, 2e-2)])
def test_gradients_of_a_student(dtype, tol):
    model, teacher, params, s, contexts, targets, w = _setup(dtype)
    with s:
        rows = s.all_params()
        torch.cuda.synchronize()
        with torch.cuda.stream(s.main):
            lists = teacher.teach(params, contexts, top=8)
            losses = model.gradients(s.models(), s.g, contexts, targets, lists, share=0.7)
        got = s.gradient()
        assert lists.value.shape == (3, 24, 8)
    for i in range(3):
        at = torch.tensor(w[i][:, :3].astype(np.int64))
        t = torch.log_softmax(_logits(teacher, params.cpu().double(), at), 1)
        best = torch.argsort(-t, dim=1, stable=True)[:, :8]
        assert torch.equal(lists.index[i].cpu().long(), best)
        row = torch.tensor(rows[i], dtype=torch.float64, requires_grad=True)
        log_p = torch.log_softmax(_logits(model, row, at), 1)
        listed = torch.zeros_like(t, dtype=torch.bool).scatter(1, best, True)
        q, left = t.exp(), torch.where(listed, 0.0, t.exp()).sum(1)
        kl = torch.where(listed, q * (t - log_p), 0.0).sum(1) + left * (left.log() - torch.logsumexp(torch.where(listed, -math.inf, log_p), 1))
        loss = 0.7 * kl.mean() + 0.3 * torch.nn.functional.nll_loss(log_p, torch.tensor(w[i][:, 3].astype(np.int64)))
        loss.backward()
        want = row.grad.numpy()
        assert abs(float(losses[i]) - float(loss.detach())) <= max(1e-5, tol if dtype == torch.bfloat16 else 0.0)
        assert np.linalg.norm(got[i] - want) <= tol * np.linalg.norm(want)


def test_a_student_steps_in_a_session():
    model, teacher, params, s, contexts, targets, _ = _setup()
    with s:
        with torch.cuda.stream(s.main):
            lists = teacher.teach(params, contexts, top=8)
        for _ in range(6):
            losses, norms = model.step(s, contexts, targets, 1.0, lists)
        s.sync()
        assert bool(torch.isfinite(losses).all()) and bool(torch.isfinite(norms).all()) and np.isfinite(s.params(-1)).all()


def _search(model, row, context, count, beams, eos, penalty):
    """The same search in 64 bits, hypothesis by hypothesis."""
    live = [(0.0, [], False)]
    for _ in range(count):
        rows = []
        for i, (score, said, ended) in enumerate(live):
            n = len(said) if not ended else said.index(eos) + 1
            if ended:
                rows.append((score / max(n, 1) ** penalty, i, 0, score, said + [eos], True))
                continue
            window = (context + said)[-CONTEXT:]
            lp = torch.log_softmax(_logits(model, row, torch.tensor([window]))[0], 0)
            for v in range(VOCAB):
                rows.append(((score + float(lp[v])) / (n + 1) ** penalty, i, v, score + float(lp[v]), said + [v], v == eos))
        rows.sort(key=lambda r: (-r[0], r[1], r[2]))
        live = [(r[3], r[4], r[5]) for r in rows[:beams]]
    return live


@pytest.mark.parametrize("beams,eos,penalty", [(1, -1, 0.0), (4, -1, 0.0), (5, 9, 0.6)])
def test_search(beams, eos, penalty):
    model, _, _, s, contexts, _, w = _setup()
    with s:
        row = s.params(-1)
        said, b = model.search(s.z[: model.d], contexts[0, :4].contiguous(), 6, beams, eos=eos, length_penalty=penalty)
        s.sync()
    for r in range(4):
        want = _search(model, torch.tensor(row, dtype=torch.float64), w[0, r, :3].tolist(), 6, beams, eos, penalty)
        assert said[r].tolist() == [x[1] for x in want]
        assert np.allclose(b.score[r].cpu().numpy(), [x[0] for x in want], rtol=0, atol=1e-4)


def test_search_in_eight_bits():
    """Logits of quantised weights are within what their rounding leaves (a step is 1 / 127 of a row's or channel's largest value), and the
    search over them is that of the model they make."""
    model, _, _, s, contexts, _, w = _setup()
    with s:
        q = model.int8(s.z[: model.d])
        at = contexts[:1].contiguous()
        plain, eight = model.logits(model.matrices(s.z[None, : model.d]), at), model.int8_logits(q, at)
        assert float((plain - eight).norm() / plain.norm()) < 0.03
        said, b = model.search(q, at[0, :4].contiguous(), 4, 3)
        for r in range(4):
            score = 0.0
            window = w[0, r, :3].tolist()
            for v in said[r, 0].tolist():
                z = model.int8_logits(q, torch.tensor([[window[-3:]]], dtype=torch.int32, device="cuda"))[0, 0].double()
                score += float(torch.log_softmax(z, 0)[v])
                window.append(v)
            assert abs(score - float(b.score[r, 0])) <= 1e-4
        s.sync()


def test_calls_on_two_streams_at_once():
    from paper_2002_09539_amd import operators as ops
    g = torch.Generator(device="cuda").manual_seed(3)
    z = [torch.randn(n, 30011, generator=g, device="cuda").bfloat16() for n in (7, 600)]
    lists = [ops.token_logprobs(t, None, top=16) for t in z]
    x, w = [torch.randn(n, 1030, generator=g, device="cuda") for n in (20, 300)], ops.quantize_weight(torch.randn(1030, 700, generator=g, device="cuda"))
    beams = [t[: t.shape[0] // 6 * 6].view(-1, 6, 30011) if t.shape[0] >= 600 else t[None, :6].contiguous() for t in z]
    scores = [torch.randn(b.shape[:2], generator=g, device="cuda") for b in beams]

    def calls(i):
        r, d = ops.distill_loss_with_grad(z[i], lists[i].top_logprob, lists[i].top_index, torch.ones(len(z[i]), device="cuda"), rest=True)
        b = ops.beam_select(beams[i], scores[i])
        return [r.loss, d, b.score, b.token, b.parent, ops.int8_matmul(x[i], w)]
    want = [calls(0), calls(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = calls(i)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_the_command_runs(capsys, monkeypatch):
    from paper_2002_09539_amd import token_model
    monkeypatch.setattr("sys.argv", ["token_model", "--rounds", "5", "--workers", "2", "--batch", "32", "--vocab", "64", "--width", "16", "--hidden", "48", "--student", "24",
                                     "--beams", "3", "--int8"])
    token_model.main()
    out = capsys.readouterr().out
    assert "student" in out and out.count("continuation") == 3 and "nan" not in out
