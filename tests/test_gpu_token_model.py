"""The operators together: a model over tokens in the rows of a Session, its gradients against 64-bit automatic differentiation,
clipping, the steps, and one-token answers.

Tolerances: of the gradients as for the block (fp32 1e-5 of the norm, here through three more operators: 3e-5; bf16 2e-2), of the loss
1e-5 and 2e-2."""
import numpy as np
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu


def _setup(dtype, m=3, tau=2, batch=24, alt=True):
    from paper_2002_09539_amd.session import Session
    from paper_2002_09539_amd.token_model import TokenModel, text
    model = TokenModel(vocab=70, context=3, width=12, hidden=40, dtype=dtype)
    data = text(70, m * batch + 3, 5)
    w = np.lib.stride_tricks.sliding_window_view(data, 4)[: m * batch].reshape(m, batch, 4).copy()
    s = Session(m, model.d, tau, 0.5, 0.2, 0.9, overlap_buffer=alt)
    s.set_option(B.OLS_OPT_SERIALIZE, 0)     # overlapped also where the refresh is small: the buffers take turns
    s.init_params(model.init(3))
    return model, s, s.upload(w[..., :3]), s.upload(w[..., 3]), w


def _want(model, row, w):
    """Loss and gradient of one worker in 64 bits."""
    row = torch.tensor(row, dtype=torch.float64, requires_grad=True)
    p = {n: row[model.offsets[n]: model.offsets[n] + a * b].view(a, b) for n, (a, b) in model.shapes.items()}
    x = (p["table"][torch.tensor(w[:, :3].astype(np.int64))] * model.scale).reshape(len(w), -1)
    z = (torch.nn.functional.silu(x @ p["w_gate"]) * (x @ p["w_up"])) @ p["w_down"]
    loss = torch.nn.functional.cross_entropy(z, torch.tensor(w[:, 3].astype(np.int64)))
    loss.backward()
    return float(loss), row.grad.numpy()


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 3e-5), (torch.bfloat16, 2e-2)])
def test_gradients(dtype, tol):
    model, s, contexts, targets, w = _setup(dtype)
    with s:
        before = s.all_params()
        with torch.cuda.stream(s.main):
            losses = model.gradients(s.models(), s.g, contexts, targets)
        got = s.gradient()
        for i in range(s.m):
            loss, grad = _want(model, before[i], w[i])
            assert abs(float(losses[i]) - loss) <= max(1e-5, tol if dtype == torch.bfloat16 else 0.0)
            assert np.linalg.norm(got[i] - grad) <= tol * np.linalg.norm(grad)
        norms = s.clip_gradients(0.25)
        clipped = s.gradient()
        for i in range(s.m):
            n = np.linalg.norm(got[i].astype(np.float64))
            assert abs(float(norms[i]) - n) <= 1e-6 * n
            assert np.allclose(clipped[i], got[i] * min(1.0, 0.25 / n), rtol=1e-6, atol=0)


@pytest.mark.parametrize("alt", [True, False])
def test_steps_follow_the_oracle(alt):
    """Two rounds and a half with clipping, with and without the second replica buffer, against the oracle's update rules fed
    with 64-bit gradients: what the models are after it depends on where the gradients read them."""
    model, s, contexts, targets, w = _setup(torch.float32, alt=alt)

    def grad(i, k, x):
        g = _want(model, x, w[i])[1]
        return g * min(1.0, 0.5 / np.linalg.norm(g))

    with s:
        x0 = s.all_params()[0]
        for k in range(5):
            model.step(s, contexts, targets, 0.5)
        got, z = s.all_params(), s.params(-1)
    m, mu, gamma, alpha, tau = 3, 0.9, 0.2, 0.5, 2
    x = np.repeat(x0[None].astype(np.float64), m, 0)
    buf, anchor = np.zeros_like(x), x0.astype(np.float64)
    for k in range(5):
        for i in range(m):
            g = grad(i, k, x[i])
            buf[i] = mu * buf[i] + g
            x[i] -= gamma * (g + mu * buf[i])
        if (k + 1) % tau == 0:
            x -= alpha * (x - anchor)
            anchor = x.mean(0)
    assert np.linalg.norm(got - x) <= 1e-4 * np.linalg.norm(x)
    assert np.linalg.norm(z - anchor) <= 1e-4 * np.linalg.norm(anchor)


def test_training_lowers_the_loss_and_answers_follow_the_model():
    model, s, contexts, targets, w = _setup(torch.float32, batch=64)
    with s:
        first = None
        for k in range(60):
            losses, _ = model.step(s, contexts, targets, 1.0)
            s.sync()
            first = first or float(losses.mean())
        assert float(losses.mean()) < 0.5 * first
        said = model.answer(s.z[: model.d], w[0, 0, :3].tolist(), 3, top=4)
        z = s.params(-1).astype(np.float64)
    p = {n: z[model.offsets[n]: model.offsets[n] + a * b].reshape(a, b) for n, (a, b) in model.shapes.items()}
    context = w[0, 0, :3].tolist()
    for step in said:
        x = (p["table"][context[-3:]] * model.scale).reshape(-1)
        a = x @ p["w_gate"]
        logits = (a / (1 + np.exp(-a)) * (x @ p["w_up"])) @ p["w_down"]
        logp = logits - logits.max() - np.log(np.exp(logits - logits.max()).sum())
        order = np.argsort(-logp, kind="stable")
        assert step["token"] == order[0] and [i for i, _ in step["alternatives"]] == order[1:4].tolist()
        assert abs(step["logprob"] - logp[order[0]]) <= 1e-4 and abs(step["entropy"] + (np.exp(logp) * logp).sum()) <= 1e-4
        context.append(step["token"])


def test_buffers_take_turns():
    model, s, contexts, targets, _ = _setup(torch.float32)
    with s:
        seen = []
        for _ in range(6):
            seen.append(B.ols_params_buffer(s.h))
            model.step(s, contexts, targets, 1.0)
        assert seen[0] == 0 and 1 in seen
        with torch.cuda.stream(s.main):
            model.gradients(s.models(), s.g, contexts, targets)
        s.local_step()
        with torch.cuda.stream(s.main):
            model.gradients(s.models(), s.g, contexts, targets)
        s.local_step()                       # tau = 2: its write is deferred
        with pytest.raises(B.OlsError):
            s.models()
        s.sync_pull()
        s.models()
