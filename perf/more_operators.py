"""Operators that turn a trained anchor into a model that answers, as measurable cases: distillation from a teacher's top
logits (loss and gradient), beam search's selection with the reordering of states, and the matrix product in 8-bit integers
with a scale for every token and every channel.

Activations and weights are normal with the variances of a network at its start, logits of a model that is neither sure nor
lost, a teacher's logits near its student's.  Where `own` is false the operators are computed in elementary torch operations
in 32 bits (in 64 where a choice or a rounding hangs on it), otherwise by the framework's kernels; `exact` is the definition
in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NONE = -math.inf


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # A few positions of an online student: launch latency.
        dict(name="distill_small", op="distill", n=16, vocab=32000, k=32, temperature=2.0, rest=False, hard=False, masked=False, dtype="bf16"),
        # Stored lists of 17 log probabilities; the teacher's remaining mass counts; padding, forbidden tokens, an odd vocabulary.
        dict(name="distill_rest_ragged", op="distill", n=1531, vocab=32003, k=17, temperature=1.0, rest=True, hard=True, masked=True, dtype="f32"),
        # A training batch: softened lists of the 32 best and the text's own tokens, loss and gradient.
        dict(name="distill_large", op="distill", n=8192, vocab=50001, k=32, temperature=2.0, rest=False, hard=True, masked=False, dtype="bf16"),
        # Long lists with the remaining mass on a large vocabulary: the largest work of this operator.
        dict(name="distill_rest_large", op="distill", n=4096, vocab=128000, k=100, temperature=1.0, rest=True, hard=False, masked=False, dtype="bf16"),
        # One request with four hypotheses and its short states: launch latency.
        dict(name="beam_serve", op="beam", batch=1, beams=4, vocab=32000, penalty=0.0, masked=False, ended=False, caches=2, length=32, width=512, dtype="bf16"),
        # Seven requests of odd sizes in mid search: hypotheses that ended, slots not yet used, forbidden tokens, scores by length.
        dict(name="beam_ragged", op="beam", batch=7, beams=5, vocab=32003, penalty=0.7, masked=True, ended=True, caches=1, length=33, width=131, dtype="f32"),
        # A serving batch on a large vocabulary: the logits are most of the bytes.
        dict(name="beam_batch", op="beam", batch=64, beams=8, vocab=128000, penalty=1.0, masked=False, ended=True, caches=2, length=1, width=1024, dtype="bf16"),
        # Long states behind a moderate vocabulary: moving them is most of the bytes.
        dict(name="beam_states", op="beam", batch=32, beams=4, vocab=50001, penalty=0.0, masked=False, ended=True, caches=4, length=128, width=1024, dtype="bf16"),
        # One token's logits from 32 000 channels: the weights are all there is to read.
        dict(name="int8_serve", op="int8", m=1, n=1, width=2048, out=32000, gated=False, dtype="bf16"),
        # Three workers with weights of their own, no dimension a whole number of tiles, in fp32.
        dict(name="int8_ragged", op="int8", m=3, n=201, width=517, out=1131, gated=False, dtype="f32"),
        # A serving batch of 64 rows through the second product of a gated block, its activation included.
        dict(name="int8_gated_batch", op="int8", m=1, n=64, width=5632, out=2048, gated=True, dtype="bf16"),
        # Scoring of long texts: the largest product.
        dict(name="int8_large", op="int8", m=1, n=8192, width=4096, out=4096, gated=False, dtype="bf16"),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """A layer's size: mostly a multiple of 8, sometimes any number."""
    v = _log_int(rng, low, high)
    return v if rng.random() < 0.3 else max(8, v // 8 * 8)


def draw(rng):
    """One more case: an operator, then sizes spread over the range in which the listed ones lie."""
    op = rng.choice(["distill", "beam", "int8"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "distill":
        c = dict(op=op, n=_log_int(rng, 1, 8192), vocab=_log_int(rng, 10, 128000), k=_log_int(rng, 1, 128), temperature=rng.choice([0.7, 1.0, 1.0, 2.0, 4.0]),
                 rest=rng.random() < 0.5, hard=rng.random() < 0.5, masked=rng.random() < 0.4, dtype=dtype)
        c["k"] = min(c["k"], c["vocab"])
        while c["n"] * c["vocab"] > (500_000_000 if dtype == "bf16" else 250_000_000):
            c["n"] //= 2
        return c
    if op == "beam":
        c = dict(op=op, batch=_log_int(rng, 1, 64), beams=_log_int(rng, 1, 16), vocab=_log_int(rng, 40, 128000), penalty=rng.choice([0.0, 0.0, 0.7, 1.0]),
                 masked=rng.random() < 0.4, ended=rng.random() < 0.6, caches=rng.choice([1, 2, 4]), length=_log_int(rng, 1, 128), width=_size(rng, 8, 1024), dtype=dtype)
        while c["batch"] * c["beams"] * c["vocab"] > 60_000_000 or c["batch"] * c["beams"] * c["caches"] * c["length"] * c["width"] > 60_000_000:
            c["batch"] = c["batch"] // 2
        return c
    c = dict(op=op, m=rng.choice([1, 1, 1, 2, 3, 5]), n=_log_int(rng, 1, 8192), width=_size(rng, 32, 8192), out=_size(rng, 16, 32000), gated=False, dtype=dtype)
    c["gated"] = dtype == "bf16" and rng.random() < 0.3
    while c["m"] * c["n"] * c["width"] * c["out"] > 1.3e11 and c["n"] > 1:
        c["n"] //= 2
    while c["m"] > 1 and c["m"] * c["width"] * c["out"] > 150_000_000:
        c["m"] -= 1
    return c


# ------------------------------------------------------------------------------------------------------------------
# what a user's program has in hand
# ------------------------------------------------------------------------------------------------------------------
class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g, device="cuda") * std).to(dtype)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def integers(self, low, high, *shape):
        return torch.randint(low, high, shape, generator=self.g, device="cuda", dtype=torch.int32)

    def tokens(self, vocab, *shape):
        """Ids by a Zipf-like law: P(v) = log((v + 2) / (v + 1)) / log(vocab + 1)."""
        u = torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float64)
        return ((vocab + 1.0) ** u - 1).floor().clamp(0, vocab - 1).to(torch.int32)


def prepare(case, seed):
    r, dt, op = _Random(seed), DTYPES[case["dtype"]], case["op"]
    s = dict(case=case)
    if op == "distill":
        n, vocab, k = case["n"], case["vocab"], case["k"]
        z = r.normal(n, vocab, std=2.5)
        s["targets"] = r.tokens(vocab, n) if case["hard"] else None
        if case["masked"]:
            forbidden = r.uniform(n, vocab) < 0.2             # by a grammar that teacher and student know
            if case["hard"]:
                forbidden.scatter_(1, s["targets"].long()[:, None], False)
            z[forbidden] = NONE
        value, index = [], []
        for i in range(0, n, 1024):                           # the teacher's lists: near the student, no two rows alike
            part = z[i: i + 1024]
            t = part + r.normal(*part.shape, std=0.8)
            v, at = torch.topk(t, k, dim=1)
            if case["rest"]:
                v = v - torch.logsumexp(t.double(), 1, keepdim=True).float()
            index.append(torch.where(v > NONE, at, -1).to(torch.int32))
            value.append(v)
        s["value"], s["index"] = torch.cat(value), torch.cat(index)
        if case["masked"] and n > 3:
            z[1] = NONE                                       # nothing is allowed here, to the teacher neither
            s["value"][1], s["index"][1] = NONE, -1
            s["value"][2], s["index"][2] = NONE, -1           # padding: neither a list nor a target
            if case["hard"]:
                s["targets"][1:3] = -1
        s["logits"] = z.to(dt)
        s["d_loss"] = 0.5 / n * (0.5 + r.uniform(n))          # weights of positions
        s["d_logprob"] = torch.full((n,), -0.5 / n, device="cuda") if case["hard"] else None
    elif op == "beam":
        batch, beams, vocab = case["batch"], case["beams"], case["vocab"]
        z = r.normal(batch, beams, vocab, std=2.5)
        if case["masked"]:
            z[r.uniform(batch, beams, vocab) < 0.2] = NONE
        s["logits"] = z.to(dt)
        s["length"] = r.integers(5, 60, batch, beams)
        s["score"] = r.normal(batch, beams) - 1.5 * s["length"]
        if case["penalty"] == 0.0:
            s["score"] = r.normal(batch, beams) - 60.0        # compared as they are: of like sizes
        s["finished"] = None
        s["eos"] = -1
        if case["ended"]:
            s["eos"] = 2
            s["finished"] = r.uniform(batch, beams) < 0.2
            if beams > 2:
                s["score"][batch // 2, beams // 2:] = NONE    # a search that has only begun
        shape = (batch, beams, case["length"], case["width"])
        s["states"] = [r.integers(0, vocab, batch, beams, 64)] + [r.normal(*shape, dtype=dt) for _ in range(case["caches"])]
        s["next"] = [torch.empty_like(t) for t in s["states"]]    # states live in two buffers that take turns
    else:
        m, n, width, out = case["m"], case["n"], case["width"], case["out"]
        s["x"] = r.normal(m, n, width, dtype=dt)
        s["up"] = r.normal(m, n, width, dtype=dt) if case["gated"] else None
        w = r.normal(m, out, width, std=width ** -0.5)
        s["w_scale"] = w.abs().amax(2) / 127
        q = torch.zeros(m, out, -(-width // 16) * 16, dtype=torch.int8, device="cuda")    # laid out once: a channel's row begins on 16 bytes
        q[:, :, :width] = torch.round(w / s["w_scale"][..., None]).clamp(-127, 127)
        s["w"] = q[:, :, :width]
    return s


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2002_09539_amd import operators as ops
    c = s["case"]
    if c["op"] == "distill":
        r, d = ops.distill_loss_with_grad(s["logits"], s["value"], s["index"], s["d_loss"], targets=s["targets"], d_logprob=s["d_logprob"],
                                          temperature=c["temperature"], rest=c["rest"])
        return {"loss": r.loss, "d_logits": d, **({"logprob": r.logprob} if c["hard"] else {})}
    if c["op"] == "beam":
        b = ops.beam_select(s["logits"], s["score"], finished=s["finished"], length=s["length"], eos=s["eos"], length_penalty=c["penalty"])
        ops.beam_reorder(s["states"], b.parent, out=s["next"])
        return {"score": b.score, "token": b.token, "parent": b.parent, "finished": b.finished, "length": b.length, "states": s["next"]}
    return {"y": ops.int8_matmul(s["x"], ops.Int8Weight(s["w"], s["w_scale"]), up=s["up"], act="silu")}


def _run_plain(s):
    return {"distill": _plain_distill, "beam": _plain_beam, "int8": _plain_int8}[s["case"]["op"]](s, s["case"])


def _plain_distill(s, c):
    z, T = s["logits"].float(), c["temperature"]
    index = s["index"].long()
    real = (index >= 0) & (index < c["vocab"])
    at = torch.where(real, index, 0)
    v = torch.where(real, s["value"], NONE)
    listed_any = real.any(1, keepdim=True)
    if c["rest"]:
        q = torch.exp(v.double())
        log_q = v
        rest = torch.where(listed_any, (1 - q.sum(1, keepdim=True)).clamp(min=0), 0.0).float()    # next to nothing: 64 bits
        q = q.float()
    else:
        u = v / T
        top = u.amax(1, keepdim=True)
        u = u - torch.where(top > NONE, top, 0.0)
        total = torch.exp(u).sum(1, keepdim=True)
        q = torch.where(total > 0, torch.exp(u) / total, 0.0)
        log_q = u - torch.log(total)
        rest = torch.zeros_like(total)
    top = z.amax(1, keepdim=True)
    empty = top == NONE
    d = z - torch.where(empty, 0.0, top)
    e = torch.exp(d / T)
    total = e.sum(1, keepdim=True)
    log_p = (d / T).gather(1, at) - torch.log(total)
    loss = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1, keepdim=True)
    weight = q.sum(1, keepdim=True) + rest
    p = e / total
    # a listed entry takes its q off, the others share the rest
    d_u = p * weight
    if c["rest"]:
        others = e.scatter(1, at, torch.where(real, 0.0, e.gather(1, at)))
        if c["masked"]:                                       # lists may hold an id -1, whose place 0 could be another entry's
            others = others * _unlisted(at, real, others)
        left = others.sum(1, keepdim=True)
        held = (rest > 0) & (left > 0)
        weight = torch.where(held, weight, weight - rest)
        loss = loss + torch.where(held, rest * (torch.log(rest) - (torch.log(left) - torch.log(total))), 0.0)
        d_u = p * weight - torch.where(held, rest * others / left, 0.0)
    d_u.scatter_add_(1, at, torch.where(real, -q, 0.0))
    grad = torch.where(empty, 0.0, d_u * (T * s["d_loss"][:, None]))
    loss = torch.where(empty & (q.sum(1, keepdim=True) == 0), 0.0, loss)
    r = {"loss": T * T * loss[:, 0]}
    if c["hard"]:
        t = s["targets"].long()
        e1 = torch.exp(d)
        total1 = e1.sum(1, keepdim=True)
        given = d.gather(1, t.clamp(min=0)[:, None])[:, 0] - torch.log(total1[:, 0])
        r["logprob"] = torch.where(t >= 0, torch.where(empty[:, 0], NONE, given), 0.0)
        g = torch.where((t >= 0) & ~empty[:, 0], s["d_logprob"], 0.0)[:, None]
        grad = grad - torch.where(empty, 0.0, g * e1 / total1)
        grad.scatter_add_(1, t.clamp(min=0)[:, None], g)
    r["d_logits"] = grad.to(s["logits"].dtype)
    return r


def _unlisted(at, real, like):
    hits = torch.zeros_like(like)
    hits.scatter_add_(1, at, real.to(like.dtype))
    return (hits == 0).to(like.dtype)


def _plain_beam(s, c):
    batch, beams, vocab = c["batch"], c["beams"], c["vocab"]
    z = s["logits"].double()                                  # which of two comes first hangs on the last bits
    top = z.amax(2, keepdim=True)
    d = z - torch.where(top > NONE, top, 0.0)
    score = s["score"].double()
    alive = score > NONE
    ended = s["finished"] & alive if s["finished"] is not None else torch.zeros_like(alive)
    raw = score[..., None] + (d - torch.log(torch.exp(d).sum(2, keepdim=True)))
    raw = torch.where((alive & ~ended)[..., None] & (z > NONE), raw, NONE)
    raw[..., 0] = torch.where(ended, score, raw[..., 0])      # an ended hypothesis stays as it is: one candidate
    key = raw
    length = s["length"]
    after = torch.where(ended, length, length + 1)
    if c["penalty"]:
        key = raw / (after.clamp(min=1).double() ** c["penalty"])[..., None]
    order = torch.sort(key.view(batch, -1), dim=1, descending=True, stable=True)
    flat = order.indices[:, :beams]
    some = order.values[:, :beams] > NONE
    own_slot = torch.arange(beams, device="cuda").expand(batch, beams)
    parent = torch.where(some, flat // vocab, own_slot)
    was = ended.gather(1, parent)
    token = torch.where(some, torch.where(was, s["eos"], flat % vocab), -1)
    new = torch.where(some, raw.view(batch, -1).gather(1, flat), NONE)
    for t, o in zip(s["states"], s["next"]):
        o.copy_(t[torch.arange(batch, device="cuda")[:, None], parent])
    return {"score": new.float(), "token": token.to(torch.int32), "parent": parent.to(torch.int32),
            "finished": some & (was | (token == s["eos"])) if s["eos"] >= 0 else some & was,
            "length": torch.where(some, after.gather(1, parent), length.gather(1, parent)).to(torch.int32), "states": s["next"]}


def _plain_int8(s, c):
    x = s["x"].float()
    if c["gated"]:                                            # next to the border between two steps: 64 bits
        a = s["x"].double()
        x = (a / (1 + torch.exp(-a)) * s["up"].double()).float()
    scale = (x.abs().amax(2, keepdim=True).double() / 127).float()
    q = torch.round(x.double() / torch.where(scale > 0, scale, 1.0).double()).float()
    acc = torch.matmul(q, s["w"].float().transpose(1, 2).contiguous())
    return {"y": (acc * scale * s["w_scale"][:, None]).to(s["x"].dtype)}


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "distill":
        n, vocab = case["n"], case["vocab"]
        return {"bytes": n * (2 * vocab * b + 8 * case["k"] + 8 + (12 if case["hard"] else 0)), "flops": n * vocab * (20 if case["hard"] else 12)}
    if case["op"] == "beam":
        rows = case["batch"] * case["beams"]
        state = 4 * 64 + case["caches"] * case["length"] * case["width"] * b
        return {"bytes": rows * (case["vocab"] * b + 2 * state + 26), "flops": 6 * rows * case["vocab"]}
    m, n, width, out = case["m"], case["n"], case["width"], case["out"]
    return {"bytes": m * (n * width * b * (2 if case["gated"] else 1) + out * (width + 4) + n * out * b), "flops": 2 * m * n * width * out}


# ------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "distill":
        parts = [_exact_distill(s, case, slice(i, i + 512)) for i in range(0, case["n"], 512)]
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return _exact_beam(s, case) if case["op"] == "beam" else _exact_int8(s, case)


def _exact_distill(s, case, rows):
    z, T, vocab = s["logits"][rows].double(), case["temperature"], case["vocab"]
    n, device = z.shape[0], z.device
    index, value = s["index"][rows].long(), s["value"][rows].double()
    inside = (index >= 0) & (index < vocab)
    where = torch.where(inside, index, vocab)                 # one column more, for what is none
    if case["rest"]:
        q = torch.where(inside, torch.exp(value), 0.0)
        log_q = value
        rest = torch.where(inside.any(1), torch.clamp(1 - q.sum(1), min=0), 0.0)
    else:
        u = torch.where(inside, value / T, NONE)
        log_q = torch.log_softmax(u, 1)
        q = torch.where(torch.isnan(log_q), 0.0, torch.exp(log_q))
        rest = torch.zeros(n, dtype=torch.float64, device=device)
    dense = torch.zeros(n, vocab + 1, dtype=torch.float64, device=device).scatter_add_(1, where, q)[:, :vocab]
    member = torch.zeros(n, vocab + 1, dtype=torch.bool, device=device).scatter_(1, where, True)[:, :vocab]
    log_p = torch.log_softmax(z / T, 1)
    none = torch.isnan(log_p[:, 0]) & (z.amax(1) == NONE)     # nothing is allowed
    log_p = torch.where(none[:, None], NONE, log_p)
    there = torch.gather(torch.cat([log_p, torch.zeros(n, 1, dtype=torch.float64, device=device)], 1), 1, where)
    loss = torch.where(q > 0, q * (log_q - there), 0.0).sum(1)
    p = torch.exp(log_p)
    total = q.sum(1)
    grad = p * total[:, None] - dense
    if case["rest"]:
        log_left = torch.logsumexp(torch.where(member, NONE, log_p), 1)
        counts = (rest > 0) & (log_left > NONE)
        loss = loss + torch.where(counts, torch.xlogy(rest, rest) - rest * torch.where(counts, log_left, 0.0), 0.0)
        share = torch.where(member, 0.0, torch.exp(log_p - torch.where(counts, log_left, 0.0)[:, None]))
        grad = grad + torch.where(counts, rest, 0.0)[:, None] * (p - share)
    grad = grad * (T * s["d_loss"][rows].double())[:, None]
    grad[none] = 0.0
    r = {"loss": T * T * loss}
    if case["hard"]:
        t = s["targets"][rows].long()
        given = t >= 0
        plain = torch.log_softmax(z, 1)
        lp = plain[torch.arange(n, device=device), t.clamp(min=0)]
        lp = torch.where(none, NONE, lp)
        r["logprob"] = torch.where(given, lp, 0.0)
        g = s["d_logprob"][rows].double() * (given & ~none)
        soft = torch.exp(plain)
        soft[none] = 0.0
        grad -= g[:, None] * soft
        grad[torch.arange(n, device=device), t.clamp(min=0)] += g
    r["d_logits"] = grad
    return r


def _exact_beam(s, case):
    batch, beams, vocab = case["batch"], case["beams"], case["vocab"]
    out = {k: [] for k in ("score", "token", "parent", "finished", "length")}
    for b in range(batch):
        lp = torch.log_softmax(s["logits"][b].double(), 1)
        candidates = []
        for i in range(beams):
            score, length = float(s["score"][b, i]), int(s["length"][b, i])
            if score == NONE:
                continue
            if s["finished"] is not None and bool(s["finished"][b, i]):
                candidates.append((score / length ** case["penalty"], i, 0, score, True, length))
                continue
            ok = torch.argsort(-lp[i], stable=True)[:beams]
            for v, t in zip(lp[i, ok].tolist(), ok.tolist()):
                if v > NONE:
                    candidates.append(((score + v) / (length + 1) ** case["penalty"], i, t, score + v, False, length + 1))
        candidates.sort(key=lambda e: (-e[0], e[1], e[2]))
        rows = candidates[:beams]
        rows = [(e[3], s["eos"] if e[4] else e[2], e[1], e[4] or e[2] == s["eos"], e[5]) for e in rows]
        rows += [(NONE, -1, i, False, int(s["length"][b, i])) for i in range(len(rows), beams)]
        for k, column in zip(out, zip(*rows)):
            out[k].append(column)
    types = dict(score=torch.float64, token=torch.int32, parent=torch.int32, finished=torch.bool, length=torch.int32)
    r = {k: torch.tensor(v, dtype=types[k], device="cuda") for k, v in out.items()}
    r["states"] = []
    for t in s["states"]:
        moved = torch.stack([t[b].index_select(0, r["parent"][b]) for b in range(batch)])
        r["states"].append(moved.double() if moved.is_floating_point() else moved)
    return r


def _exact_int8(s, case):
    y = []
    for w in range(case["m"]):
        x = s["x"][w].double()
        if case["gated"]:
            x = x * torch.sigmoid(x) * s["up"][w].double()
        scale = (x.abs().amax(1) / 127).float().double()      # a scale is a 32-bit number
        q = torch.where(scale[:, None] > 0, x / scale[:, None], 0.0).round()
        y.append((q @ s["w"][w].double().T) * scale[:, None] * s["w_scale"][w].double())
    return {"y": torch.stack(y)}
