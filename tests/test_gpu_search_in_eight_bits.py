"""The token model's search with weights in 8 bits is the search over the model that they make: the logits are those of int8_logits, the
choice is made in 64 bits, hypothesis by hypothesis."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

VOCAB, CONTEXT, WIDTH, HIDDEN = 70, 3, 12, 40


def _search(model, q, context, count, beams, eos, penalty):
    """(score, tokens said, whether it has ended) of the best, best first."""
    live = [(0.0, [], False)]
    for _ in range(count):
        windows = [(context + said)[-CONTEXT:] for _, said, _ in live]
        z = model.int8_logits(q, torch.tensor([windows], dtype=torch.int32, device="cuda"))[0]
        lp = torch.log_softmax(z.double(), 1).cpu()
        rows = []
        for i, (score, said, ended) in enumerate(live):
            if ended:
                rows.append((score / (said.index(eos) + 1) ** penalty, i, 0, score, said + [eos], True))
                continue
            for v in range(VOCAB):
                s = score + float(lp[i, v])
                rows.append((s / (len(said) + 1) ** penalty, i, v, s, said + [v], v == eos))
        rows.sort(key=lambda r: (-r[0], r[1], r[2]))
        live = [r[3:] for r in rows[:beams]]
    return live


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("beams,eos,penalty", [(1, -1, 0.0), (4, -1, 0.0), (5, 9, 0.6), (6, 3, 1.0)])
def test_search_over_quantised_weights(beams, eos, penalty, dtype):
    from paper_2002_09539_amd.token_model import TokenModel
    model = TokenModel(VOCAB, CONTEXT, WIDTH, HIDDEN, dtype=dtype)
    q = model.int8(torch.from_numpy(model.init(3)).cuda() * 1.5)
    contexts = torch.randint(0, VOCAB, (5, CONTEXT), generator=torch.Generator().manual_seed(beams), dtype=torch.int32)
    said, b = model.search(q, contexts.cuda(), 5, beams, eos=eos, length_penalty=penalty)
    for r in range(5):
        want = _search(model, q, contexts[r].tolist(), 5, beams, eos, penalty)
        assert said[r].tolist() == [w[1] for w in want]
        assert b.finished[r].tolist() == [w[2] for w in want]
        assert b.length[r].tolist() == [w[1].index(eos) + 1 if w[2] else 5 for w in want]
        # sums of five logarithms, each good to 1e-6, and of roundings of the score between steps
        assert np.allclose(b.score[r].cpu().numpy(), [w[0] for w in want], rtol=2.0 ** -21, atol=1e-5)
