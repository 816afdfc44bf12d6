"""A small model over tokens, trained by Overlap Local-SGD with the operators of token models, and asked for its next token.

Every worker holds an embedding table and a gated feed-forward block whose output width is the vocabulary: the `context`
last tokens' embeddings, side by side, go through the block, and its outputs are the logits of the next token.

    gradients   embed -> gated_ffn -> token_logprobs_with_grad -> gated_ffn_grad -> embed_grad, into the rows of g
    step        Session.clip_gradients, local_step, and every tau-th time sync_pull and anchor_update_async
    answer      the anchor, one token at a time: embed -> gated_ffn -> token_logprobs with alternatives
    student     a model that learns from the anchor's lists of best tokens as well: token_logprobs of the anchor, then
                distill_loss_with_grad in the place of token_logprobs_with_grad
    search      several continuations at once, scored as a whole: embed -> gated_ffn -> beam_select -> beam_reorder, with the weights as they
                are or in 8 bits (quantize_weight once, then int8_matmul twice in the place of gated_ffn)

    python -m paper_2002_09539_amd.token_model [--rounds 30] [--dtype bf16] [--student 128] [--beams 4] [--int8]

trains eight workers on synthetic text (each on its own share of it, not shuffled) and prints the loss and an answer.
"""
import argparse
from collections import namedtuple

import numpy as np
import torch

from . import operators as ops
from .session import Session


Int8Model = namedtuple("Int8Model", "table gate_up down")
Lists = namedtuple("Lists", "value index")        # a teacher's best tokens of every position: log probabilities and ids


class TokenModel:
    """The model of every worker of a Session, at the front of its parameter rows.

    dtype: the activations'.  bfloat16 rounds the fp32 master weights on the way into the products."""

    def __init__(self, vocab, context, width, hidden, act="silu", dtype=torch.float32):
        self.vocab, self.context, self.width, self.hidden, self.act, self.dtype = vocab, context, width, hidden, act, dtype
        self.shapes = dict(table=(vocab, width), w_gate=(context * width, hidden), w_up=(context * width, hidden), w_down=(hidden, vocab))
        self.offsets, at = {}, 0
        for name, shape in self.shapes.items():
            self.offsets[name] = at
            at += -(-shape[0] * shape[1] // 8) * 8          # every matrix on a 16-byte boundary of its bf16 or fp32 row
        self.d = at
        self.scale = width ** 0.5                            # the table is small at the start, its rows are not

    def init(self, seed):
        """[d] fp32, the same for every worker: normal with the variance that keeps activations at one."""
        r = np.random.Generator(np.random.Philox(key=seed))
        x = np.zeros(self.d, dtype=np.float32)
        for name, shape in self.shapes.items():
            at = self.offsets[name]
            std = shape[1] ** -0.5 if name == "table" else shape[0] ** -0.5
            x[at: at + shape[0] * shape[1]] = r.standard_normal(shape[0] * shape[1], dtype=np.float32) * np.float32(std)
        return x

    def matrices(self, rows):
        """Views [m][..][..] of the matrices in parameter or gradient rows [m][ld]."""
        return {n: rows[:, self.offsets[n]: self.offsets[n] + s[0] * s[1]].unflatten(1, s) for n, s in self.shapes.items()}

    def logits(self, p, contexts, save=False):
        """contexts: int32 [m][B][context] -> logits [m][B][vocab] (and x, saved for the backward pass)."""
        m, batch = contexts.shape[:2]
        x = ops.embed(p["table"], contexts, self.scale, dtype=self.dtype).view(m, batch, self.context * self.width)
        if not save:
            return ops.gated_ffn(x, p["w_gate"], p["w_up"], p["w_down"], self.act)
        y, saved = ops.gated_ffn(x, p["w_gate"], p["w_up"], p["w_down"], self.act, save=True)
        return y, x, saved

    def teach(self, params, contexts, top=32):
        """Lists of the `top` best tokens behind each of contexts [..., context], by one model's parameters [d]."""
        z = self.logits(self.matrices(params[None]), contexts.reshape(1, -1, self.context))
        r = ops.token_logprobs(z, None, top=top)
        return Lists(*(t.view(*contexts.shape[:-1], top) for t in (r.top_logprob, r.top_index)))

    def gradients(self, rows, g, contexts, targets, lists=None, share=0.5):
        """Writes the gradients of the mean negative log likelihood, per worker, into g [m][ld]; returns the losses [m].

        lists: a teacher's, of [m][B] positions; the loss is then `share` of the divergence from them and 1 - share of the likelihood."""
        m, batch = targets.shape
        p, out = self.matrices(rows), self.matrices(g)
        z, x, saved = self.logits(p, contexts, save=True)
        each = torch.full((m, batch), -1.0 / batch, device=z.device)
        if lists is None:
            r, dz = ops.token_logprobs_with_grad(z, targets, each, out=z)
            loss = -r.logprob.mean(1)
        else:
            r, dz = ops.distill_loss_with_grad(z, lists.value, lists.index, each * -share, targets=targets, d_logprob=each * (1 - share), rest=True, out=z)
            loss = share * r.loss.mean(1) - (1 - share) * r.logprob.mean(1)
        into = ops.FfnGrads(None, out["w_gate"], out["w_up"], out["w_down"])
        dx = ops.gated_ffn_grad(dz, x, p["w_gate"], p["w_up"], p["w_down"], saved, self.act, out=into).x
        ops.embed_grad(contexts, dx.view(m, batch, self.context, self.width), self.vocab, self.scale, out=out["table"], workers=m)
        return loss

    def step(self, s, contexts, targets, max_norm, lists=None, share=0.5):
        """One iteration of all workers of the Session; returns their losses and the norms of their gradients."""
        with torch.cuda.stream(s.main):
            losses = self.gradients(s.models(), s.step_g, contexts, targets, lists, share)
        norms = s.clip_gradients(max_norm)
        s.run(1)
        return losses, norms

    def answer(self, params, context, count, top=5):
        """`count` tokens after `context` (a list), each the likeliest, by one model's parameters [d]; with each the log
        probability, the entropy and the alternatives."""
        p = self.matrices(params[None])
        context, said = list(context), []
        for _ in range(count):
            ids = torch.tensor([[context[-self.context:]]], dtype=torch.int32, device=params.device)
            r = ops.token_logprobs(self.logits(p, ids), None, top=top)
            best = [(int(i), float(v)) for i, v in zip(r.top_index.flatten(), r.top_logprob.flatten())]
            said.append(dict(token=best[0][0], logprob=best[0][1], entropy=float(r.entropy), alternatives=best[1:]))
            context.append(best[0][0])
        return said


    def int8(self, params):
        """One model's parameters [d] with its products' weights in 8 bits, laid out for search()."""
        p = self.matrices(params[None])
        return Int8Model(p["table"], ops.quantize_weight(torch.cat([p["w_gate"], p["w_up"]], 2)), ops.quantize_weight(p["w_down"]))

    def int8_logits(self, q, contexts):
        """logits() by an Int8Model: both first projections in one product, the activation on the way into the second."""
        m, batch = contexts.shape[:2]
        x = ops.embed(q.table, contexts, self.scale, dtype=self.dtype).view(m, batch, self.context * self.width)
        ab = ops.int8_matmul(x, q.gate_up)
        return ops.int8_matmul(ab[..., : self.hidden], q.down, up=ab[..., self.hidden:], act=self.act)

    def search(self, params, contexts, count, beams=4, eos=-1, length_penalty=0.0):
        """The best `beams` continuations of `count` tokens behind contexts, int32 [batch][context], by one model's parameters [d] or an
        Int8Model: (tokens [batch][beams][count], Beams), best first; behind a token `eos` a continuation has ended and repeats it."""
        batch, device = contexts.shape[0], contexts.device
        p = params if isinstance(params, Int8Model) else self.matrices(params[None])
        logits = self.int8_logits if isinstance(params, Int8Model) else self.logits
        window = contexts[:, None].repeat(1, beams, 1)
        said = torch.full((batch, beams, count), -1, dtype=torch.int32, device=device)
        score = torch.full((batch, beams), -torch.inf, device=device)
        score[:, 0] = 0.0                                    # one hypothesis at first
        b = ops.Beams(score, None, None, torch.zeros(batch, beams, dtype=torch.bool, device=device), torch.zeros(batch, beams, dtype=torch.int32, device=device))
        for i in range(count):
            z = logits(p, window.view(1, batch * beams, self.context)).view(batch, beams, self.vocab)
            b = ops.beam_select(z, b.score, finished=b.finished, length=b.length, eos=eos, length_penalty=length_penalty)
            ops.beam_reorder([window, said], b.parent)
            window = torch.cat([window[..., 1:], b.token[..., None]], 2)
            said[..., i] = b.token
        return said, b


def text(vocab, length, seed):
    """Synthetic text: most tokens follow from the two before, the others are drawn by a Zipf-like law."""
    r = np.random.Generator(np.random.Philox(key=seed))
    drawn = np.minimum((vocab + 1.0) ** r.uniform(size=length), vocab).astype(np.int64) - 1
    told = r.uniform(size=length) < 0.7
    t = drawn.copy()
    for i in range(2, length):
        if told[i]:
            t[i] = (5 * t[i - 1] + 3 * t[i - 2] + 1) % vocab
    return t.astype(np.int32)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--tau", type=int, default=4)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=512)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="f32")
    ap.add_argument("--student", type=int, default=0, help="hidden units of a second model that learns from the first one's anchor")
    ap.add_argument("--beams", type=int, default=0, help="answer by a search over this many continuations, too")
    ap.add_argument("--int8", action="store_true", help="search with weights in 8 bits")
    a = ap.parse_args()
    m, context, nb = a.workers, 2, 16
    model = TokenModel(a.vocab, context, a.width, a.hidden, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype])
    data = text(a.vocab, m * nb * a.batch + context, 1)
    windows = np.lib.stride_tricks.sliding_window_view(data, context + 1)[: m * nb * a.batch].reshape(m, nb, a.batch, context + 1).copy()
    with Session(m, model.d, a.tau, 0.5, 0.5, 0.9) as s:
        contexts, targets = s.upload(windows[..., :context]), s.upload(windows[..., context])
        s.init_params(model.init(2))
        for k in range(a.rounds * a.tau):
            losses, norms = model.step(s, contexts[:, k % nb], targets[:, k % nb], 1.0)
            if (k + 1) % (5 * a.tau) == 0:
                s.sync()
                print("iteration %4d  loss %.4f  gradient norm before clipping %.3f" % (k + 1, float(losses.mean()), float(norms.mean())), flush=True)
        s.sync()
        for said in model.answer(s.z[: model.d], data[:context].tolist(), 4):
            print("token %4d  log probability %.3f  entropy %.3f  also %s" % (said["token"], said["logprob"], said["entropy"], said["alternatives"][:2]))
        teacher, params = model, s.z[: model.d].clone()
        torch.cuda.synchronize()
    if a.student:
        model = TokenModel(a.vocab, context, a.width, a.student, dtype=model.dtype)
        with Session(m, model.d, a.tau, 0.5, 0.5, 0.9) as s:
            contexts, targets = s.upload(windows[..., :context]), s.upload(windows[..., context])
            with torch.cuda.stream(s.main):
                lists = teacher.teach(params, contexts)
            s.init_params(model.init(3))
            for k in range(a.rounds * a.tau):
                losses, norms = model.step(s, contexts[:, k % nb], targets[:, k % nb], 1.0, Lists(lists.value[:, k % nb], lists.index[:, k % nb]))
                if (k + 1) % (5 * a.tau) == 0:
                    s.sync()
                    print("student    %4d  loss %.4f" % (k + 1, float(losses.mean())), flush=True)
            s.sync()
            params = s.z[: model.d].clone()
            torch.cuda.synchronize()
    if a.beams:
        start = torch.from_numpy(data[:context][None].copy()).to(params.device)
        said, b = model.search(model.int8(params) if a.int8 else params, start, 6, a.beams)
        for tokens, score in zip(said[0].tolist(), b.score[0].tolist()):
            print("continuation %s  log probability %.3f" % (tokens, score))


if __name__ == "__main__":
    main()
