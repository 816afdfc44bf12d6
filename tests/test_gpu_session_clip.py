"""Session.clip_gradients scales what the next local step reads, and nothing else.

A step without momentum is x - gamma g, one fp32 product and sum (2^-23 each), of a clipped element (2^-22): 1e-6 of the sum of sizes."""
import numpy as np
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

M, D, GAMMA = 3, 1000, 0.25


def _session(**kw):
    from paper_2002_09539_amd.session import Session
    s = Session(M, D, kw.pop("tau", 4), 0.5, GAMMA, 0.0, **kw)
    s.init_params(np.zeros(D, dtype=np.float32))
    return s


def _gradient(s, seed):
    g = torch.zeros(M, s.ld, device="cuda")
    g[:, :D] = torch.randn(M, D, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    torch.cuda.synchronize()
    return g


def _check_step(s, before, max_norm, norms):
    want = before[:, :D].double().cpu().numpy()
    length = np.linalg.norm(want, axis=1)
    assert np.allclose(norms.double().cpu().numpy(), length, rtol=1e-6)
    s.run(1)
    assert np.allclose(s.all_params(), -GAMMA * want * np.minimum(1.0, max_norm / length)[:, None], rtol=1e-6, atol=1e-9)


@pytest.mark.parametrize("own", [True, False])
def test_gradients_of_set_gradient(own):
    with _session(own_gradient=own) if own else _unbound() as s:
        mine, other = _gradient(s, 1), _gradient(s, 2)
        before, kept = other.clone(), mine.clone()
        if own:
            s.g.copy_(mine)
        torch.cuda.synchronize()
        s.set_gradient(other)
        norms = s.clip_gradients(2.0)
        s.sync()
        _check_step(s, before, 2.0, norms)
        if own:
            assert torch.equal(s.g, kept)


def _unbound():
    from paper_2002_09539_amd.session import Session
    s = Session(M, D, 4, 0.5, GAMMA, 0.0, own_gradient=False)
    with pytest.raises(B.OlsError):
        s.clip_gradients(1.0)
    s.bind(_gradient(s, 9))
    s.init_params(np.zeros(D, dtype=np.float32))
    return s


def test_bound_gradients():
    with _session() as s:
        g = _gradient(s, 3)
        s.g.copy_(g)
        torch.cuda.synchronize()
        norms = s.clip_gradients(1.0)
        s.sync()
        _check_step(s, g, 1.0, norms)


def test_gradients_that_a_deferred_step_needs_are_left_alone():
    with _session(tau=1) as s:
        g = _gradient(s, 4)
        s.g.copy_(g)
        torch.cuda.synchronize()
        s.local_step()                                   # tau = 1: its write is deferred
        with pytest.raises(B.OlsError):
            s.clip_gradients(1e-3)
        s.sync_pull()
        s.anchor_update_async()
        s.sync()
        assert torch.equal(s.g, g)
        s.clip_gradients(1e-3)


def test_an_attached_model_writes_its_own():
    from paper_2002_09539_amd.session import Session
    with Session(M, 12 * 8 + 8 + 8 * 4 + 4, 4, 0.5, GAMMA, 0.0) as s:
        s.attach_mlp((12, 8, 4), 16)
        with pytest.raises(B.OlsError):
            s.clip_gradients(1.0)
