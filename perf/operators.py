"""The operators of token models, as measurable cases: embedding lookup and its gradient, log probabilities of given
tokens with entropy and top alternatives (and their gradient), the gated feed-forward block forward and backward, and
gradient clipping by global norm.

Each runs for m workers at once, as everything here does (m = 1 is an ordinary call).  Ids of tokens follow a Zipf-like
law, as words do; activations and weights are normal with the variances of a network at its start.  Where `own` is false
the operators are computed in elementary torch operations in 32 bits, otherwise by the framework's kernels; `exact` is
the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # One decoding step of a serving batch: a row for each of 64 sequences; launch latency.
        dict(name="embed_serve", op="embed", m=1, vocab=32000, width=1024, n=64, dtype="bf16", grad=""),
        # Four workers of the ragged kind: odd vocabulary and width, padded sequences; gradient rows in fp32.
        dict(name="embed_grad_ragged", op="embed_grad", m=4, vocab=5003, width=389, n=1201, dtype="f32", grad="f32"),
        # A training batch of 32 k tokens on a large vocabulary: the gradient table is most of the bytes.
        dict(name="embed_grad_large", op="embed_grad", m=1, vocab=50001, width=1024, n=32768, dtype="bf16", grad="f32"),
        # A few sequences being sampled: what was chosen, how sure the model was, and what else it might have said.
        dict(name="logprob_serve", op="logprob", m=1, vocab=128000, n=4, dtype="f32", top=8, masked=False),
        # Scoring of given answers, some tokens forbidden (-inf), with the five best alternatives.
        dict(name="logprob_score", op="logprob", m=1, vocab=32003, n=1531, dtype="bf16", top=5, masked=True),
        # The training loss: likelihood and an entropy bonus, with the gradient at the logits.
        dict(name="logprob_train", op="logprob_train", m=1, vocab=50001, n=8192, dtype="bf16", top=0, masked=False),
        # Clipping the gradients of a small model: 40 tensors, one norm; latency.
        dict(name="clip_small", op="clip", m=1, tensors=40, total=300_000, dtype="f32"),
        # Sixteen workers, each with a norm of its own, at the size of configuration 3's parameter vectors.
        dict(name="clip_workers", op="clip", m=16, tensors=16, total=16 * 14_700_000, dtype="f32"),
        # One token through a gated block: the weights are all there is to read.
        dict(name="ffn_serve", op="ffn", m=1, n=1, width=2048, hidden=5632, out=2048, act="silu", dtype="bf16"),
        # Three small workers with no dimension a whole number of tiles, forward and backward in fp32.
        dict(name="ffn_train_ragged", op="ffn_train", m=3, n=201, width=300, hidden=517, out=131, act="gelu", dtype="f32"),
        # Two workers' mini-batches of 1024 rows, forward and backward.
        dict(name="ffn_train_workers", op="ffn_train", m=2, n=1024, width=1024, hidden=2816, out=1024, act="silu", dtype="bf16"),
        # A training step of a large block: the largest work.
        dict(name="ffn_train_large", op="ffn_train", m=1, n=8192, width=2048, hidden=5632, out=2048, act="silu", dtype="bf16"),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """A layer's size: mostly a multiple of 8, sometimes any number."""
    v = _log_int(rng, low, high)
    return v if rng.random() < 0.3 else max(8, v // 8 * 8)


def draw(rng):
    """One more case: an operator, then sizes spread over the range in which the listed ones lie."""
    op = rng.choice(["embed", "embed_grad", "logprob", "logprob_train", "clip", "ffn", "ffn_train"])
    dtype = rng.choice(["f32", "bf16"])
    m = rng.choice([1, 1, 2, 3, 5, 8])
    if op in ("embed", "embed_grad"):
        c = dict(op=op, m=m, vocab=_log_int(rng, 300, 128000), width=_size(rng, 32, 2048), n=_log_int(rng, 1, 32768),
                 dtype=dtype, grad=rng.choice(["f32", dtype]) if op == "embed_grad" else "")
        while c["m"] * c["vocab"] * c["width"] > 60_000_000:
            c["m"], c["vocab"] = max(1, c["m"] // 2), max(300, c["vocab"] // 2)
        while c["m"] * c["n"] * c["width"] > 40_000_000:
            c["n"] //= 2
        return c
    if op in ("logprob", "logprob_train"):
        c = dict(op=op, m=m, vocab=_log_int(rng, 10, 128000), n=_log_int(rng, 1, 8192), dtype=dtype,
                 top=rng.choice([0, 1, 5, 8, 20]) if op == "logprob" else 0, masked=rng.random() < 0.4)
        c["top"] = min(c["top"], c["vocab"])
        while c["m"] * c["n"] * c["vocab"] > (60_000_000 if c["top"] else 200_000_000) and c["n"] > 1:
            c["n"] //= 2
        return c
    if op == "clip":
        return dict(op=op, m=m, tensors=m * _log_int(rng, 1, 100), total=_log_int(rng, 1000, 150_000_000), dtype=dtype)
    c = dict(op=op, m=m, n=_log_int(rng, 1, 8192), width=_size(rng, 32, 2048), hidden=_size(rng, 32, 5632),
             out=_size(rng, 16, 2048), act=rng.choice(["silu", "gelu", "relu"]), dtype=dtype)
    most = 1.5e11 if dtype == "bf16" else 2e10
    while c["m"] * c["n"] * c["hidden"] * (2 * c["width"] + c["out"]) > most and c["n"] > 1:
        c["n"] //= 2
    return c


# ------------------------------------------------------------------------------------------------------------------
# what a user's program has in hand
# ------------------------------------------------------------------------------------------------------------------
class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g, device="cuda") * std).to(dtype)

    def tokens(self, vocab, *shape):
        """Ids by a Zipf-like law: P(v) = log((v + 2) / (v + 1)) / log(vocab + 1)."""
        u = torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float64)
        return ((vocab + 1.0) ** u - 1).floor().clamp(0, vocab - 1).to(torch.int32)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")


def _sizes(case):
    """Element counts of a model's tensors, each worker's like the others': sizes spread over three decades."""
    each = case["tensors"] // case["m"]
    weight = np.exp(np.random.RandomState(each).uniform(0, 7, each))
    total = case["total"] // case["m"]
    return [max(1, int(total * w / weight.sum())) for w in weight] * case["m"]


def prepare(case, seed):
    r, dt, m = _Random(seed), DTYPES[case["dtype"]], case["m"]
    op = case["op"]
    s = dict(case=case)
    if op in ("embed", "embed_grad"):
        n, width = case["n"], case["width"]
        t = r.tokens(case["vocab"], m, n)
        s["scale"] = math.sqrt(width)
        if n > 100:
            t[:, n - n // 16:] = -1          # the padding at a batch's end
        s["tokens"] = t
        if op == "embed":
            s["table"] = r.normal(m, case["vocab"], width, std=0.02, dtype=dt)
        else:
            s["d_out"] = r.normal(m, n, width, std=1e-3, dtype=dt)
    elif op in ("logprob", "logprob_train"):
        rows, vocab = m * case["n"], case["vocab"]
        z = r.normal(rows, vocab, std=2.5)
        s["targets"] = r.tokens(vocab, rows)
        if case["masked"]:
            z[r.uniform(rows, vocab) < 0.2] = -math.inf     # tokens that a grammar forbids
            z.scatter_(1, s["targets"].long()[:, None], 1.0)  # the given one is allowed
            if rows > 2:
                z[1] = -math.inf                             # a finished sequence: nothing is allowed
                s["targets"][2] = -1                         # a position without a target
        s["logits"] = z.to(dt)
        if op == "logprob_train":
            s["d_logprob"] = torch.full((rows,), -1.0 / rows, device="cuda")
            s["d_entropy"] = -0.01 / rows * r.uniform(rows)
    elif op == "clip":
        s["grads"] = [r.normal(k, std=1e-2, dtype=dt) for k in _sizes(case)]
        pitch = [-(-g.numel() // 64) * 64 for g in s["grads"]]      # one buffer for all, each tensor on a line of its own
        s["flat"] = torch.zeros(sum(pitch), dtype=dt, device="cuda")
        s["out"] = [o[: g.numel()] for o, g in zip(s["flat"].split(pitch), s["grads"])]
        per = case["tensors"] // m
        s["groups"] = [i // per for i in range(len(s["grads"]))]
        s["of"] = torch.tensor(s["groups"], device="cuda")
        s["max_norm"] = 0.5 * 1e-2 * math.sqrt(case["total"] / m)
    else:
        n, width, hidden, out = case["n"], case["width"], case["hidden"], case["out"]
        s["x"] = r.normal(m, n, width, dtype=dt)
        s["w_gate"] = r.normal(m, width, hidden, std=width ** -0.5, dtype=dt)
        s["w_up"] = r.normal(m, width, hidden, std=width ** -0.5, dtype=dt)
        s["w_down"] = r.normal(m, hidden, out, std=hidden ** -0.5, dtype=dt)
        if op == "ffn_train":
            s["dy"] = r.normal(m, n, out, std=1e-2, dtype=dt)
    return s


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2002_09539_amd import operators as ops
    c = s["case"]
    op = c["op"]
    if op == "embed":
        return {"out": ops.embed(s["table"], s["tokens"], s["scale"])}
    if op == "embed_grad":
        return {"grad": ops.embed_grad(s["tokens"], s["d_out"], c["vocab"], s["scale"], dtype=DTYPES[c["grad"]], workers=c["m"])}
    if op == "logprob":
        r = ops.token_logprobs(s["logits"], s["targets"], top=c["top"])
        return _named(r, c["top"])
    if op == "logprob_train":
        r, d = ops.token_logprobs_with_grad(s["logits"], s["targets"], s["d_logprob"], s["d_entropy"])
        return {**_named(r, 0), "d_logits": d}
    if op == "clip":
        norms = ops.clip_grad_norm(s["grads"], s["max_norm"], groups=s["groups"], out=s["out"])
        return {"norms": norms, "out": s["flat"]}
    if op == "ffn":
        return {"y": ops.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], c["act"])}
    y, saved = ops.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], c["act"], save=True)
    g = ops.gated_ffn_grad(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"], saved, c["act"])
    return {"y": y, "dx": g.x, "dw_gate": g.w_gate, "dw_up": g.w_up, "dw_down": g.w_down}


def _named(r, top):
    d = {"logprob": r.logprob, "entropy": r.entropy, "logsumexp": r.logsumexp}
    if top:
        d.update(top_logprob=r.top_logprob, top_index=r.top_index)
    return d


def _act(name, a):
    if name == "silu":
        return a * torch.sigmoid(a)
    if name == "gelu":
        return 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    return torch.where(a > 0, a, torch.zeros_like(a))


def _act_grad(name, a):
    if name == "silu":
        g = torch.sigmoid(a)
        return g * (1 + a * (1 - g))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    return (a > 0).to(a.dtype)


def _run_plain(s):
    c = s["case"]
    op, m, dt = c["op"], c["m"], DTYPES[c["dtype"]]
    if op in ("embed", "embed_grad"):
        t = s["tokens"].long()
        real = (t >= 0) & (t < c["vocab"])
        first = torch.arange(m, device="cuda")[:, None] * c["vocab"]
        if op == "embed":
            rows = s["table"].view(-1, c["width"])[(first + t.clamp(0, c["vocab"] - 1))].float()
            return {"out": torch.where(real[..., None], rows * s["scale"], 0.0).to(dt)}
        grad = torch.zeros(m * c["vocab"], c["width"], device="cuda")
        grad.index_add_(0, (first + t)[real], s["d_out"][real].float() * s["scale"])
        return {"grad": grad.view(m, c["vocab"], c["width"]).to(DTYPES[c["grad"]])}
    if op in ("logprob", "logprob_train"):
        z = s["logits"].float()
        t = s["targets"].long()
        top = z.amax(1, keepdim=True)
        empty = top == -math.inf
        z0 = z - torch.where(empty, 0.0, top)
        e = torch.exp(z0)
        total = e.sum(1, keepdim=True)
        lse0 = torch.log(total)
        logp = z0 - lse0                                        # nan in an empty row
        p = e / total
        plogp = torch.where(p > 0, p * logp, 0.0)
        entropy = -plogp.sum(1, keepdim=True)
        given = torch.where(t >= 0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        none = empty[:, 0]
        r = {"logprob": torch.where(none & (t >= 0), -math.inf, given), "entropy": torch.where(none, 0.0, entropy[:, 0]),
             "logsumexp": torch.where(none, -math.inf, (top + lse0)[:, 0])}
        if op == "logprob":
            if c["top"]:
                v, i = torch.sort(z, dim=1, descending=True, stable=True)
                v, i = v[:, : c["top"]], i[:, : c["top"]]
                gone = v == -math.inf
                r["top_logprob"] = torch.where(gone, -math.inf, logp.gather(1, i))
                r["top_index"] = torch.where(gone, -1, i).to(torch.int32)
            return r
        glp = torch.where(t >= 0, s["d_logprob"], 0.0)[:, None]
        d = -glp * p - s["d_entropy"][:, None] * (plogp + p * entropy)
        d = torch.where(empty, 0.0, torch.where(p > 0, d, 0.0))
        d.scatter_add_(1, t.clamp(min=0)[:, None], torch.where(empty, 0.0, glp))
        return {**r, "d_logits": d.to(dt)}
    if op == "clip":
        squares = torch.stack([g.float().square().sum() for g in s["grads"]])
        norms = torch.zeros(m, device="cuda").index_add_(0, s["of"], squares).sqrt()
        k = torch.where(norms > s["max_norm"], s["max_norm"] / norms, 1.0)
        for g, o, i in zip(s["grads"], s["out"], s["groups"]):
            o.copy_(g.float() * k[i])
        return {"norms": norms, "out": s["flat"]}
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    a, b = torch.matmul(x, wg), torch.matmul(x, wu)
    g = _act(c["act"], a)
    h = g * b
    y = torch.matmul(h, wd)
    if op == "ffn":
        return {"y": y.to(dt)}
    dy = s["dy"].float()
    dh = torch.matmul(dy, wd.transpose(1, 2).contiguous())
    da, db = dh * b * _act_grad(c["act"], a), dh * g
    ht, xt = h.transpose(1, 2).contiguous(), x.transpose(1, 2).contiguous()
    dx = torch.matmul(da, wg.transpose(1, 2).contiguous()) + torch.matmul(db, wu.transpose(1, 2).contiguous())
    return {"y": y.to(dt), "dx": dx.to(dt), "dw_gate": torch.matmul(xt, da).to(dt), "dw_up": torch.matmul(xt, db).to(dt),
            "dw_down": torch.matmul(ht, dy).to(dt)}


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def _bytes(dtype):
    return 4 if dtype == "f32" else 2


def _distinct(vocab, n):
    """Expected number of distinct ids among n of them."""
    v = np.arange(vocab, dtype=np.float64)
    p = np.log1p(1.0 / (v + 1)) / math.log(vocab + 1)
    return float(-np.expm1(n * np.log1p(-p)).sum())


def work(case):
    op, m, b = case["op"], case["m"], _bytes(case["dtype"])
    if op in ("embed", "embed_grad"):
        n, width = case["n"], case["width"]
        rows = n - (n // 16 if n > 100 else 0)
        if op == "embed":
            return {"bytes": m * (n * width * b + _distinct(case["vocab"], rows) * width * b + 4 * n), "flops": m * n * width}
        return {"bytes": m * (rows * width * b + case["vocab"] * width * _bytes(case["grad"]) + 4 * n), "flops": 2 * m * rows * width}
    if op in ("logprob", "logprob_train"):
        rows, vocab = m * case["n"], case["vocab"]
        if op == "logprob":
            return {"bytes": rows * (vocab * b + 16 + 8 * case["top"]), "flops": 6 * rows * vocab}
        return {"bytes": rows * (2 * vocab * b + 24), "flops": 14 * rows * vocab}
    if op == "clip":
        return {"bytes": 2 * b * sum(_sizes(case)), "flops": 3 * sum(_sizes(case))}
    n, width, hidden, out = case["n"], case["width"], case["hidden"], case["out"]
    weights, acts = 2 * width * hidden + hidden * out, n * (width + out)
    products = 2 * n * weights
    if op == "ffn":
        return {"bytes": m * b * (weights + acts), "flops": m * products}
    return {"bytes": m * b * (2 * weights + 2 * acts), "flops": 3 * m * products}


# ------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op, m = case["op"], case["m"]
    if op == "embed":
        rows = []
        for w in range(m):
            t = s["tokens"][w].long()
            keep = ((t >= 0) & (t < case["vocab"])).double()[:, None]
            rows.append(s["table"][w].index_select(0, t * (keep[:, 0] > 0)).double() * keep * s["scale"])
        return {"out": torch.stack(rows)}
    if op == "embed_grad":
        tables = []
        for w in range(m):
            t = s["tokens"][w].long()
            keep = torch.nonzero((t >= 0) & (t < case["vocab"]))[:, 0]
            g = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
            tables.append(g.index_put_((t[keep],), s["d_out"][w][keep].double() * s["scale"], accumulate=True))
        return {"grad": torch.stack(tables)}
    if op in ("logprob", "logprob_train"):
        parts = [_exact_rows(s, case, slice(i, i + 1024)) for i in range(0, m * case["n"], 1024)]
        return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    if op == "clip":
        norm = [0.0] * m
        for g, i in zip(s["grads"], s["groups"]):
            norm[i] += float(torch.linalg.vector_norm(g.double())) ** 2
        norm = [math.sqrt(v) for v in norm]
        whole = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
        at = 0
        for g, i in zip(s["grads"], s["groups"]):
            whole[at: at + g.numel()] = g.double() * min(1.0, s["max_norm"] / norm[i] if norm[i] else 1.0)
            at += -(-g.numel() // 64) * 64
        return {"norms": torch.tensor(norm, dtype=torch.float64), "out": whole}
    y, dx, dg, du, dd = [], [], [], [], []
    for w in range(m):
        x, wg, wu, wd = (s[k][w].double() for k in ("x", "w_gate", "w_up", "w_down"))
        a, b = x @ wg, x @ wu
        if case["act"] == "silu":
            sig = 1 / (1 + torch.exp(-a))
            f, df = a * sig, sig + a * sig * (1 - sig)
        elif case["act"] == "gelu":
            cdf = 0.5 * torch.erfc(-a / math.sqrt(2))
            f, df = a * cdf, cdf + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
        else:
            f, df = a.clamp(min=0), (a > 0).double()
        y.append((f * b) @ wd)
        if op == "ffn":
            continue
        dy = s["dy"][w].double()
        dh = dy @ wd.T
        dd.append((f * b).T @ dy)
        da, db = dh * b * df, dh * f
        dg.append(x.T @ da)
        du.append(x.T @ db)
        dx.append(da @ wg.T + db @ wu.T)
    if op == "ffn":
        return {"y": torch.stack(y)}
    return {"y": torch.stack(y), "dx": torch.stack(dx), "dw_gate": torch.stack(dg), "dw_up": torch.stack(du), "dw_down": torch.stack(dd)}


def _exact_rows(s, case, rows):
    z, t = s["logits"][rows].double(), s["targets"][rows].long()
    n = z.shape[0]
    at = torch.arange(n, device="cuda")
    lse = torch.logsumexp(z, 1)
    some = lse > -math.inf
    logp = torch.log_softmax(z, 1)
    p = logp.exp()
    surprise = torch.where(p > 0, -logp * p, torch.zeros_like(p))
    entropy = surprise.sum(1)
    lp = logp[at, t.clamp(min=0)]
    lp[~some] = -math.inf
    lp[t < 0] = 0.0
    r = {"logprob": lp, "entropy": torch.where(some, entropy, torch.zeros_like(entropy)), "logsumexp": lse}
    if case["op"] == "logprob":
        if case["top"]:
            i = torch.argsort(-z, dim=1, stable=True)[:, : case["top"]]
            v = logp[at[:, None], i]
            gone = z[at[:, None], i] == -math.inf
            v[gone], i[gone] = -math.inf, -1
            r.update(top_logprob=v, top_index=i.to(torch.int32))
        return r
    hot = torch.zeros_like(z)
    hot[at, t.clamp(min=0)] = 1.0
    w = (s["d_logprob"][rows].double() * (t >= 0))[:, None]
    d = w * (hot - p) + s["d_entropy"][rows].double()[:, None] * (surprise - p * entropy[:, None])
    d[~some] = 0.0
    r["d_logits"] = d
    return r
