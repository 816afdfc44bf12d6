"""Operators of token models on torch tensors: embedding lookup, gated feed-forward block, log probabilities, clipping, distillation,
beam search, products in 8-bit integers.

Each function checks its tensors, allocates its results and workspace, and enqueues libols kernels on torch's current
stream of the tensors' device (see the section of the same name in include/ols.h).  Nothing synchronises and nothing is
kept.  Tensors are fp32 or bf16, ids int32.  A leading axis of m workers can stand in front of every tensor, so that
weights and gradients can be views of the rows of a Session's x and g; rows may be strided, elements of a row may not.
Tensors that were made on another stream are the caller's to order and to record, as with any torch operation.

Nothing here takes part in automatic differentiation: results carry no graph, also where a tensor requires gradients, and so end any
graph that leads to them.  Every operator has a function for its gradient, which the caller calls.
"""
import contextlib
from array import array
from collections import namedtuple

import torch

from . import binding as B

TokenLogprobs = namedtuple("TokenLogprobs", "logprob entropy logsumexp top_logprob top_index stats")

_DTYPE = {torch.float32: B.OLS_F32, torch.bfloat16: B.OLS_BF16}


def _refuse(message, *args):
    raise B.OlsError(B.OLS_EINVAL, message % args)


def _dtype(t, name):
    code = _DTYPE.get(t if isinstance(t, torch.dtype) else t.dtype)
    if code is None:
        _refuse("%s must be float32 or bfloat16, got %s", name, t if isinstance(t, torch.dtype) else t.dtype)
    return code


def _on_gpu(first, *others):
    """The device that all tensors are on."""
    place = first.get_device()
    if place < 0:
        _refuse("tensors must be on the GPU: there is no CPU path")
    for t in others:
        if t is not None and t.get_device() != place:
            _refuse("tensors are on %s and %s", first.device, t.device)
    return first.device


_SAME = contextlib.nullcontext()


def _on(device):
    """The tensors' device as the current one, which it mostly is."""
    index = device if isinstance(device, int) else device.index
    return _SAME if index == torch._C._cuda_getDevice() else torch.cuda.device(index)


def _stream(device):
    """The handle of torch's current stream (torch.cuda.current_stream(device).cuda_stream without the object)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _rows(t, name):
    """(worker stride, row stride) of a [m][rows][width] tensor whose rows are contiguous."""
    m, rows, width = t.shape
    group, row, step = t.stride()
    if step != 1 and width > 1:
        _refuse("%s: the elements of a row must be contiguous", name)
    if m * rows * width == 0:
        return 0, max(1, width)
    return (group if m > 1 else 0), (row if rows > 1 else max(width, row))


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- embeddings ---------------------------------------------------------------------------------------------------
def _ids(tokens, m):
    if tokens.dtype != torch.int32:
        _refuse("ids must be int32, got %s", tokens.dtype)
    if m < 1:
        _refuse("at least one worker is needed, got %d", m)
    ids = tokens.reshape(m, -1) if tokens.is_contiguous() else tokens.reshape(m, -1).contiguous()
    return ids, (ids.shape[1] if m > 1 else 0)


def embed(table, tokens, scale=1.0, out=None, dtype=None):
    """out[..., :] = scale * table[tokens]; ids outside [0, vocab) give rows of zeros.

    table: [vocab, width] with tokens of any shape, or [m, vocab, width] with tokens [m, ...].  The result is
    tokens.shape + (width,), of `dtype` (the table's by default) or in `out`."""
    if table.dim() not in (2, 3):
        _refuse("a table is [vocab, width] or [m, vocab, width], got %d axes", table.dim())
    device = _on_gpu(table, tokens, out)
    workers = table.dim() == 3
    m = table.shape[0] if workers else 1
    if workers and (tokens.dim() < 1 or tokens.shape[0] != m):
        _refuse("%d workers' tables with ids of shape %s", m, tuple(tokens.shape))
    t3 = table if workers else table.unsqueeze(0)
    ids, ids_group = _ids(tokens, m)
    n, (vocab, width) = ids.shape[1], t3.shape[1:]
    if out is None:
        out = torch.empty(*tokens.shape, width, dtype=dtype or table.dtype, device=device)
    elif tuple(out.shape) != (*tokens.shape, width) or not out.is_contiguous() or (dtype and out.dtype != dtype):
        _refuse("out must be a contiguous %s of the result's type", (*tokens.shape, width))
    tg, tr = _rows(t3, "table")
    with _on(device):
        B.ols_embed(m, n, vocab, width, ids.data_ptr(), ids_group, t3.data_ptr(), _dtype(table, "table"), tr, tg, float(scale), out.data_ptr(),
                    _dtype(out, "out"), width, n * width, _stream(device))
    return out


def embed_grad(tokens, d_out, vocab, scale=1.0, out=None, dtype=torch.float32, accumulate=False, workers=None):
    """The table's gradient: grad[v] = scale * sum of d_out over the positions of v, in order of position.

    tokens: any shape, d_out: tokens.shape + (width,); the result is [vocab, width], in `dtype` or in `out`.  With
    workers = m the first axis of tokens and d_out is the workers' and the result is [m, vocab, width].  out may be a view
    of gradient rows; accumulate adds to it and leaves the rows of absent ids alone."""
    device = _on_gpu(d_out, tokens, out)
    if tuple(d_out.shape[:-1]) != tuple(tokens.shape) or d_out.dim() < 1:
        _refuse("d_out of shape %s for ids of shape %s", tuple(d_out.shape), tuple(tokens.shape))
    if accumulate and out is None:
        _refuse("accumulate needs the gradient to add to")
    m = 1 if workers is None else int(workers)
    if workers is not None and (tokens.dim() < 1 or tokens.shape[0] != m):
        _refuse("ids of shape %s for %d workers", tuple(tokens.shape), m)
    ids, ids_group = _ids(tokens, m)
    n, width = ids.shape[1], d_out.shape[-1]
    d3 = d_out if d_out.dim() == 3 and workers is not None else d_out.reshape(m, n, width)
    shape = (vocab, width) if workers is None else (m, vocab, width)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device)
    elif tuple(out.shape) != shape:
        _refuse("out must be of shape %s, got %s", shape, tuple(out.shape))
    o3 = out.unsqueeze(0) if workers is None else out
    dg, dr = _rows(d3, "d_out")
    og, orow = _rows(o3, "out")
    nbytes = B.ols_embed_grad_workspace_bytes(m, n, vocab, width)
    with _on(device):
        ws = _workspace(nbytes, device)
        B.ols_embed_grad(m, n, vocab, width, ids.data_ptr(), ids_group, d3.data_ptr(), _dtype(d_out, "d_out"), dr, dg, float(scale), out.data_ptr(),
                         _dtype(out, "out"), orow, og, int(accumulate), _ptr(ws), nbytes, _stream(device))
    return out


# ---- gated feed-forward block -------------------------------------------------------------------------------------
FfnGrads = namedtuple("FfnGrads", "x w_gate w_up w_down")

_ACT = {"silu": B.OLS_ACT_SILU, "gelu": B.OLS_ACT_GELU, "relu": B.OLS_ACT_RELU}


def _matrix(t, m, shape, name):
    """A tensor as the C boundary takes it: [m][rows][cols], without the worker axis [rows][cols] shared by the workers."""
    have, stride = t.shape, t.stride()
    rows, width = shape
    group = 0
    if have != shape or not (m == 1 or name in _SHARED):
        if have != (m, rows, width):
            _refuse("%s must be of shape %s, got %s", name, (m, *shape), tuple(have))
        group = stride[0] if m > 1 else 0
    if stride[-1] != 1 and width > 1:
        _refuse("%s: the elements of a row must be contiguous", name)
    if 0 in have:
        return B.ols_matrix(t.data_ptr(), max(1, width), 0)
    row = stride[-2]
    return B.ols_matrix(t.data_ptr(), row if rows > 1 or row > width else width, group)


def _saved(t):
    """Address and bytes of what a forward call left."""
    if t.dtype != torch.uint8 or t.dim() != 1 or not t.is_contiguous():
        _refuse("saved must be what gated_ffn(..., save=True) returned")
    return (t.data_ptr() if t.numel() else None), t.numel()


_SHARED = ("x", "w_gate", "w_up", "w_down", "dy", "up", "weight")    # inputs that may come without a worker axis


def _ffn(x, w_gate, w_up, w_down, act, others):
    device = _on_gpu(x, w_gate, w_up, w_down, *others)
    if act not in _ACT:
        _refuse("unknown activation %r: one of %s", act, ", ".join(_ACT))
    if x.dim() not in (2, 3) or w_gate.dim() not in (2, 3):
        _refuse("x is [rows, width] or [m, rows, width], weights [width, hidden] or [m, width, hidden]")
    workers = x.dim() == 3 or w_gate.dim() == 3
    m = x.shape[0] if x.dim() == 3 else w_gate.shape[0] if workers else 1
    rows, width, hidden, out = x.shape[-2], x.shape[-1], w_gate.shape[-1], w_down.shape[-1]
    if w_gate.dtype != w_up.dtype or w_gate.dtype != w_down.dtype:
        _refuse("the weights must share one type")
    f = B.ols_ffn()
    f.groups, f.act, f.dtype, f.weight_dtype = m, _ACT[act], _dtype(x, "x"), _dtype(w_gate, "the weights")
    f.grad_dtype = f.weight_dtype
    f.rows, f.width, f.hidden, f.out = rows, width, hidden, out
    f.x = _matrix(x, m, (rows, width), "x")
    f.w_gate = _matrix(w_gate, m, (width, hidden), "w_gate")
    f.w_up = _matrix(w_up, m, (width, hidden), "w_up")
    f.w_down = _matrix(w_down, m, (hidden, out), "w_down")
    return f, device, ((m,) if workers else ())


def gated_ffn(x, w_gate, w_up, w_down, act="silu", save=False, out=None):
    """y = (act(x w_gate) * (x w_up)) w_down; act: "silu", "gelu" (by the error function) or "relu".

    x: [rows, width] or [m, rows, width]; weights: [width, hidden], [width, hidden], [hidden, out], with or without the
    workers' axis in front (without: shared).  x bf16: products of bf16 operands, weights bf16 or fp32 (rounded on the way);
    x fp32: products of fp32 accuracy, fp32 weights.  save=True returns (y, saved) for gated_ffn_grad."""
    f, device, lead = _ffn(x, w_gate, w_up, w_down, act, (out,))
    shape = (*lead, f.rows, f.out)
    with _on(device):
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=device)
        elif tuple(out.shape) != shape or out.dtype != x.dtype:
            _refuse("out must be of shape %s and x's type", shape)
        f.y = _matrix(out, f.groups, (f.rows, f.out), "out")
        saved = None
        if save:
            f.saved_bytes = B.ols_gated_ffn_saved_bytes(f)
            saved = torch.empty(f.saved_bytes, dtype=torch.uint8, device=device)
            f.saved = saved.data_ptr() if f.saved_bytes else None
        f.ws_bytes = B.ols_gated_ffn_workspace_bytes(f, 0)
        ws = _workspace(f.ws_bytes, device)
        f.ws = _ptr(ws)
        B.ols_gated_ffn(f, _stream(device))
    return (out, saved) if save else out


def gated_ffn_grad(dy, x, w_gate, w_up, w_down, saved, act="silu", out=None, grad_dtype=None, need_x=True):
    """Gradients of sum(dy * y): FfnGrads(x, w_gate, w_up, w_down), from what gated_ffn(..., save=True) left.

    The weights' gradients are of grad_dtype (the weights' type by default) and have a worker axis if anything has one: a
    shared weight's gradient is each worker's.  out: a FfnGrads of tensors to write to (views of gradient rows, say; None
    entries are allocated), of which x may be dy or x itself; need_x=False leaves out the gradient at x."""
    f, device, lead = _ffn(x, w_gate, w_up, w_down, act, (dy, saved, *(out or ())))
    if dy.dtype != x.dtype:
        _refuse("dy must be of x's type")
    f.dy = _matrix(dy, f.groups, (f.rows, f.out), "dy")
    shapes = ((f.rows, f.width), (f.width, f.hidden), (f.width, f.hidden), (f.hidden, f.out))
    if out is not None:
        types = {t.dtype for t in out[1:] if t is not None}
        if len(types) > 1 or (grad_dtype and types - {grad_dtype}):
            _refuse("the weights' gradients must share one type")
        grad_dtype = grad_dtype or (types.pop() if types else None)
    grad_dtype = grad_dtype or w_gate.dtype
    f.grad_dtype = _dtype(grad_dtype, "grad_dtype")
    with _on(device):
        made = []
        for i, (name, shape) in enumerate(zip(("dx", "g_gate", "g_up", "g_down"), shapes)):
            t = out[i] if out is not None else None
            if i == 0 and not need_x:
                made.append(None)
                continue
            dtype = x.dtype if i == 0 else grad_dtype
            if t is None:
                t = torch.empty(*lead, *shape, dtype=dtype, device=device)
            elif tuple(t.shape) != (*lead, *shape) or t.dtype != dtype:
                _refuse("out.%s must be %s of shape %s", FfnGrads._fields[i], dtype, (*lead, *shape))
            setattr(f, name, _matrix(t, f.groups, shape, name))
            made.append(t)
        f.saved, f.saved_bytes = _saved(saved)
        f.ws_bytes = B.ols_gated_ffn_workspace_bytes(f, 1)
        ws = _workspace(f.ws_bytes, device)
        f.ws = _ptr(ws)
        B.ols_gated_ffn_grad(f, _stream(device))
    return FfnGrads(*made)


# ---- log probabilities --------------------------------------------------------------------------------------------
def _logit_rows(t, name):
    shape = t.shape
    if not shape or shape[-1] < 1:
        _refuse("%s must have a last axis of tokens, got shape %s", name, tuple(shape))
    vocab = shape[-1]
    if len(shape) == 2:
        row, step = t.stride()
        if step == 1 or vocab == 1:
            return t, shape[0], row if shape[0] > 1 else vocab     # rows that overlap are refused by the boundary
    if not t.is_contiguous():
        _refuse("%s must be contiguous, or two-dimensional with contiguous rows", name)
    return t, t.numel() // vocab, vocab


def _per_row(t, shape, dtype, name):
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype:
        _refuse("%s must be %s of shape %s, got %s of shape %s", name, dtype, tuple(shape), t.dtype, tuple(t.shape))
    return t.contiguous()


def _floats(device, *shape):
    return torch.empty(*shape, dtype=torch.float32, device=device) if shape else torch.empty((), dtype=torch.float32, device=device)


def _logprobs(logits, targets, top, d_logprob, d_entropy, d_logits):
    device = _on_gpu(logits, targets, d_logprob, d_entropy, d_logits)
    z, rows, stride = _logit_rows(logits, "logits")
    shape, vocab = logits.shape[:-1], logits.shape[-1]
    code = _dtype(logits, "logits")
    targets = _per_row(targets, shape, torch.int32, "targets")
    d_logprob = _per_row(d_logprob, shape, torch.float32, "d_logprob")
    d_entropy = _per_row(d_entropy, shape, torch.float32, "d_entropy")
    d_stride = 0
    if d_logits is not None:
        if d_logits.shape != logits.shape or d_logits.dtype != logits.dtype:
            _refuse("the gradient must have the logits' shape and type")
        d_stride = _logit_rows(d_logits, "out")[2]
    top = int(top)
    nbytes = B.ols_token_logprobs_workspace_bytes(rows, vocab, code, top)
    with _on(device):
        ws = _workspace(nbytes, device)
        results = torch.empty(3, *shape, dtype=torch.float32, device=device)
        stats = torch.empty(*shape, 2, dtype=torch.float32, device=device)
        best = torch.empty(*shape, top, dtype=torch.float32, device=device) if top else None
        index = torch.empty(*shape, top, dtype=torch.int32, device=device) if top else None
        logprob, entropy, lse = results.unbind(0)
        B.ols_token_logprobs(rows, vocab, z.data_ptr(), code, stride, _ptr(targets), logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), stats.data_ptr(),
                             top, _ptr(best), _ptr(index), _ptr(d_logprob), _ptr(d_entropy), _ptr(d_logits), d_stride, _ptr(ws), nbytes, _stream(device))
    return TokenLogprobs(logprob, entropy, lse, best, index, stats)


def token_logprobs(logits, targets=None, top=0):
    """Log probability of targets[...] under logits[..., vocab], the rows' entropy and logsumexp, and the `top` best tokens.

    logits: contiguous, or two-dimensional with contiguous rows that do not overlap (an expanded row is refused).  targets: int32 of
    shape logits.shape[:-1]; one outside [0, vocab) is none (logprob 0).  Returns TokenLogprobs: logprob,
    entropy, logsumexp of that shape, top_logprob and top_index with a last axis of `top` (None with top = 0), and stats
    (the largest logit and the sum of e^(z - it), for token_logprobs_grad)."""
    return _logprobs(logits, targets, top, None, None, None)


def token_logprobs_with_grad(logits, targets, d_logprob, d_entropy=None, top=0, out=None):
    """token_logprobs and the gradient at the logits of sum(d_logprob * logprob + d_entropy * entropy), in one call.

    The gradient has the logits' type; out may be the logits themselves.  At a target whose logit is -inf it is d_logprob.  Returns (TokenLogprobs, gradient)."""
    if out is None:
        _on_gpu(logits)
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    return _logprobs(logits, targets, top, d_logprob, d_entropy, out), out


def token_logprobs_grad(logits, targets, result, d_logprob, d_entropy=None, out=None):
    """The same gradient from an earlier call's TokenLogprobs, for upstream gradients that were not known then."""
    device = _on_gpu(logits, targets, d_logprob, d_entropy, out, result.stats)
    z, rows, stride = _logit_rows(logits, "logits")
    shape, vocab = logits.shape[:-1], logits.shape[-1]
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        _refuse("the gradient must have the logits' shape and type")
    targets = _per_row(targets, shape, torch.int32, "targets")
    d_logprob = _per_row(d_logprob, shape, torch.float32, "d_logprob")
    d_entropy = _per_row(d_entropy, shape, torch.float32, "d_entropy")
    stats = _per_row(result.stats, (*shape, 2), torch.float32, "stats")
    entropy = _per_row(result.entropy, shape, torch.float32, "entropy")
    with _on(device):
        B.ols_token_logprobs_grad(rows, vocab, z.data_ptr(), _dtype(logits, "logits"), stride, _ptr(targets), stats.data_ptr(), entropy.data_ptr(),
                                  _ptr(d_logprob), _ptr(d_entropy), out.data_ptr(), _logit_rows(out, "out")[2], _stream(device))
    return out


# ---- clipping -----------------------------------------------------------------------------------------------------
def _distinct(pointers, sizes):
    """Whether no two tensors that have elements begin at one address."""
    if len(set(pointers)) == len(pointers):
        return True
    real = [p for p, n in zip(pointers, sizes) if n]
    return len(set(real)) == len(real)


def _clip(grads, max_norm, groups, out):
    grads = list(grads)
    if not grads:
        _refuse("no tensors")
    n, first = len(grads), grads[0]
    device, dtype = _on_gpu(first), first.dtype
    code = _dtype(first, "a gradient")
    out = grads if out is None else list(out)
    if len(out) != n:
        _refuse("%d outputs for %d tensors", len(out), n)
    every = grads if out is grads else grads + out
    place = first.get_device()
    if {t.dtype for t in every} != {dtype} or {t.get_device() for t in every} != {place}:
        _refuse("the tensors must share one type and one device")
    if not all([t.is_contiguous() for t in every]):
        _refuse("the tensors must be contiguous")
    sizes = [t.numel() for t in grads]
    if out is not grads and [t.numel() for t in out] != sizes:
        _refuse("outputs must have their inputs' sizes")
    order, group_array, count = None, None, 1
    if groups is not None:
        groups = list(groups)
        if len(groups) != n or min(groups) < 0:
            _refuse("every tensor needs the number of its group")
        count = max(groups) + 1
        if sorted(groups) != groups:
            order = sorted(range(n), key=groups.__getitem__)      # stable: a group's tensors keep their order
            groups, sizes = [groups[i] for i in order], [sizes[i] for i in order]
            grads, out = [grads[i] for i in order], (None if out is grads else [out[i] for i in order])
            out = grads if out is None else out
        group_array = array("i", groups)
    places = [t.data_ptr() for t in grads]
    inputs, numel, outputs = array("Q", places), array("q", sizes), None
    if max_norm is not None:
        if out is not grads:
            places = [t.data_ptr() for t in out]
        if not _distinct(places, sizes):
            _refuse("a tensor cannot be scaled twice in one call")
        outputs = inputs if out is grads else array("Q", places)
    at = lambda a: None if a is None else a.buffer_info()[0]  # noqa: E731
    nbytes = B.ols_clip_workspace_bytes(n, at(numel), at(group_array), count)
    with _on(place):
        norms = torch.empty(count, dtype=torch.float32, device=device)
        ws = _workspace(nbytes, device)
        B.ols_clip_gradients(n, at(inputs), at(outputs), at(numel), at(group_array), count, code, 0.0 if max_norm is None else float(max_norm), norms.data_ptr(),
                             _ptr(ws), nbytes, _stream(device))
    return norms


def grad_norm(grads, groups=None):
    """The 2-norm over all tensors of each group: a tensor of max(groups) + 1 norms, one without `groups`."""
    return _clip(grads, None, groups, None)


def clip_grad_norm(grads, max_norm, groups=None, out=None):
    """Scales each group's tensors by min(1, max_norm / norm), in place or into `out`; returns the norms before that.

    grads: contiguous tensors of one type; groups[i]: the number of tensor i's group (one group by default).  What is written must not
    overlap: a gradient that several parameters share is given once."""
    return _clip(grads, max_norm, groups, out)


# ---- distillation -------------------------------------------------------------------------------------------------
DistillLoss = namedtuple("DistillLoss", "loss logprob stats")


def _distill(logits, top_value, top_index, targets, d_loss, d_logprob, temperature, rest, d_logits):
    device = _on_gpu(logits, top_value, top_index, targets, d_loss, d_logprob, d_logits)
    z, rows, stride = _logit_rows(logits, "logits")
    *shape, vocab = logits.shape
    listed = top_value.shape
    shape = tuple(shape)
    if not listed or listed[:-1] != shape:
        _refuse("lists of shape %s for logits of shape %s", tuple(listed), tuple(logits.shape))
    if targets is None and d_logprob is not None:
        _refuse("a gradient of log probabilities needs the targets")
    top_value, top_index = _per_row(top_value, listed, torch.float32, "top_value"), _per_row(top_index, listed, torch.int32, "top_index")
    targets, d_loss = _per_row(targets, shape, torch.int32, "targets"), _per_row(d_loss, shape, torch.float32, "d_loss")
    d_logprob = _per_row(d_logprob, shape, torch.float32, "d_logprob")
    keep = top_value, top_index, targets, d_loss, d_logprob
    d_stride = 0
    if d_logits is logits:
        d_stride = stride
    elif d_logits is not None:
        if d_logits.shape != logits.shape or d_logits.dtype != logits.dtype:
            _refuse("the gradient must have the logits' shape and type")
        d_stride = _logit_rows(d_logits, "out")[2]
    d = B.ols_distill(_dtype(logits, "logits"), listed[-1], int(rest), float(temperature), rows, vocab, z.data_ptr(), stride, top_value.data_ptr(),
                      top_index.data_ptr(), _ptr(targets), None, None, None, _ptr(d_loss), _ptr(d_logprob), _ptr(d_logits), d_stride)
    return d, shape, device, keep


def _distill_loss(logits, top_value, top_index, targets, d_loss, d_logprob, temperature, rest, d_logits):
    d, shape, device, keep = _distill(logits, top_value, top_index, targets, d_loss, d_logprob, temperature, rest, d_logits)
    d.ws_bytes = B.ols_distill_workspace_bytes(d.rows, d.vocab, d.dtype, d.k)
    with _on(device):
        ws = _workspace(d.ws_bytes, device)
        loss, stats = _floats(device, *shape), _floats(device, *shape, 8)
        logprob = None if targets is None else _floats(device, *shape)
        d.loss, d.logprob, d.stats, d.ws = loss.data_ptr(), _ptr(logprob), stats.data_ptr(), _ptr(ws)
        B.ols_distill_loss(d, _stream(device))
    return DistillLoss(loss, logprob, stats)


def distill_loss(logits, top_value, top_index, targets=None, temperature=1.0, rest=False):
    """temperature^2 KL(teacher || student) per row, of a student's logits[..., vocab] and lists of the teacher's best tokens.

    top_value (fp32) and top_index (int32): logits.shape[:-1] + (k,), k <= 256, as token_logprobs(..., top=k) returns them; an index outside
    [0, vocab) is no entry.  rest=False: the teacher's distribution is that of the list alone, softmax(top_value / temperature).  rest=True:
    top_value are log probabilities at this temperature, and what they leave of one stands against what the student leaves outside the
    list.  targets (int32, optional): tokens whose log probability at temperature 1 is returned too.  Returns DistillLoss: loss and logprob of
    shape logits.shape[:-1] (logprob None without targets), and stats for distill_loss_grad.  A loss is good to some 2^-20 temperature^2 (a row's sums
    are fp32)."""
    return _distill_loss(logits, top_value, top_index, targets, None, None, temperature, rest, None)


def distill_loss_with_grad(logits, top_value, top_index, d_loss, targets=None, d_logprob=None, temperature=1.0, rest=False, out=None):
    """distill_loss and the gradient at the logits of sum(d_loss * loss + d_logprob * logprob), in one call.

    d_loss and d_logprob: fp32 of shape logits.shape[:-1], or None.  The gradient has the logits' type; out may be the logits themselves.
    The teacher has none.  Returns (DistillLoss, gradient)."""
    if out is None:
        _on_gpu(logits)
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    return _distill_loss(logits, top_value, top_index, targets, d_loss, d_logprob, temperature, rest, out), out


def distill_loss_grad(logits, top_value, top_index, result, d_loss, targets=None, d_logprob=None, temperature=1.0, rest=False, out=None):
    """The same gradient from an earlier call's DistillLoss (of the same lists, targets, temperature and rest), for upstream gradients that
    were not known then."""
    if (targets is None) != (result.logprob is None):
        _refuse("targets must be those of the earlier call")
    if out is None:
        _on_gpu(logits)
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    d, shape, device, keep = _distill(logits, top_value, top_index, targets, d_loss, d_logprob, temperature, rest, out)
    _on_gpu(logits, result.stats)
    stats = _per_row(result.stats, (*shape, 8), torch.float32, "stats")
    d.stats = stats.data_ptr()
    with _on(device):
        B.ols_distill_loss_grad(d, _stream(device))
    return out


# ---- beam search --------------------------------------------------------------------------------------------------
Beams = namedtuple("Beams", "score token parent finished length")


def _int32(v, name):
    """A whole number that the C boundary holds: ctypes would take others modulo 2^32."""
    v = int(v)
    if not -1 << 31 <= v < 1 << 31:
        _refuse("%s must be in [-2^31, 2^31), got %d", name, v)
    return v


def beam_select(logits, score, beams=None, finished=None, length=None, eos=-1, length_penalty=0.0):
    """The best `beams` continuations (as many as there are hypotheses by default) of each request, best first.

    logits: [batch, hypotheses, vocab], the elements of a row contiguous; score: fp32 [batch, hypotheses], the sums of log probabilities so far,
    -inf for no hypothesis.  finished (bool) and length (int32), both [batch, hypotheses] and optional: a hypothesis that has ended stays in the
    race as it is; candidates are compared by score / length ** length_penalty.  At most 32 hypotheses; ties go to the lower hypothesis,
    then to the lower token.  Returns Beams of shape [batch, beams]: score, token (eos behind an ended hypothesis, -1 in places without a
    candidate), parent (the hypothesis continued, for beam_reorder), finished, and length (None without lengths)."""
    device = _on_gpu(logits, score, finished, length)
    if logits.dim() != 3:
        _refuse("logits are [batch, hypotheses, vocab], got %d axes", logits.dim())
    (batch, have, vocab), stride = logits.shape, logits.stride()
    if vocab > 1 and stride[2] != 1:
        _refuse("logits: the elements of a row must be contiguous")
    code, beams = _dtype(logits, "logits"), have if beams is None else _int32(beams, "beams")
    rows, eos = (batch, have), _int32(eos, "eos")
    score, finished = _per_row(score, rows, torch.float32, "score"), _per_row(finished, rows, torch.bool, "finished")
    length = _per_row(length, rows, torch.int32, "length")
    nbytes = B.ols_beam_workspace_bytes(batch, have, beams, vocab, code)
    with _on(device):
        ws = _workspace(nbytes, device)
        parts = torch.empty(3 if length is None else 4, batch, beams, dtype=torch.int32, device=device).unbind(0)
        new_score, token, parent = parts[0].view(torch.float32), parts[1], parts[2]
        new_length = None if length is None else parts[3]
        ended = torch.empty(batch, beams, dtype=torch.bool, device=device)
        b = B.ols_beam(code, have, beams, eos, batch, vocab, logits.data_ptr(), stride[0], stride[1], score.data_ptr(), _ptr(finished), _ptr(length),
                       float(length_penalty), new_score.data_ptr(), token.data_ptr(), parent.data_ptr(), _ptr(new_length), ended.data_ptr(), _ptr(ws), nbytes)
        B.ols_beam_select(b, _stream(device))
    return Beams(new_score, token, parent, ended, new_length)


def _state_rows(t, batch, beams, name):
    """(bytes of a row, bytes between requests, bytes between hypotheses) of a state [batch, beams, ...]."""
    shape, size = t.shape, t.element_size()
    if len(shape) < 2:
        _refuse("%s must be [batch, hypotheses, ...], got %d axes", name, len(shape))
    if shape[0] != batch or shape[1] != beams:
        _refuse("%s is of shape %s, for %d requests of %d hypotheses", name, tuple(shape), batch, beams)
    if batch * beams == 0:
        return 0, 0, 0
    if t.is_contiguous():
        n = t.numel() // (batch * beams) * size
        return n, n * beams, n
    n = 1
    for i in range(len(shape) - 1, 1, -1):
        if shape[i] != 1 and t.stride(i) != n:
            _refuse("%s: what one hypothesis holds must be contiguous", name)
        n *= shape[i]
    return n * size, t.stride(0) * size, t.stride(1) * size


def beam_reorder(states, parent, out=None):
    """Moves hypotheses' states behind a step: state[b, i] = old state[b, parent[b, i]] for every tensor of `states`; returns the list written.

    states: tensors [batch, hypotheses, ...] of any types, what one hypothesis holds contiguous (a slice of the positions used so far is, where they
    are the first of these axes).  parent: int32 [batch, beams] (Beams.parent); one outside the hypotheses leaves its place as it was.
    Without `out` the tensors are written in place, and hypotheses that stay are not touched; `out` holds other tensors of shape
    [batch, beams, ...], which must not overlap the states or each other.  Nothing that is written may be `parent` itself."""
    states = list(states)
    if not states:
        return []
    if parent.dtype != torch.int32 or parent.dim() != 2:
        _refuse("parent must be int32 [batch, beams], got %s of shape %s", parent.dtype, tuple(parent.shape))
    outs = states if out is None else list(out)
    if len(outs) != len(states):
        _refuse("%d outputs for %d states", len(outs), len(states))
    device = _on_gpu(parent, *states, *(() if out is None else outs))
    batch, beams = parent.shape
    have = states[0].shape[1] if states[0].dim() > 1 else 0
    src, dst = [t.data_ptr() for t in states], [t.data_ptr() for t in outs]
    rows = [_state_rows(t, batch, have, "a state") for t in states]
    row_bytes, src_batch, src_beam = zip(*rows)
    if out is None:
        if have != beams:
            _refuse("in place, %d hypotheses cannot become %d", have, beams)
        dst_batch, dst_beam = src_batch, src_beam
    else:
        for s, o in zip(states, outs):
            if o.dtype != s.dtype or (o.shape != s.shape and o.shape[2:] != s.shape[2:]):
                _refuse("an output is %s of shape %s, for a state of %s and shape %s", o.dtype, tuple(o.shape), s.dtype, tuple(s.shape))
        _, dst_batch, dst_beam = zip(*[_state_rows(t, batch, beams, "an output") for t in outs])
        if not set(src).isdisjoint(dst):
            read = {}
            for i, (p, n) in enumerate(zip(src, row_bytes)):
                if n:
                    read[p] = i if p not in read else -1       # -1: a state that is read several times
            if any(n and read.get(p, i) != i for i, (p, n) in enumerate(zip(dst, row_bytes))):
                _refuse("an output is another state of the call")
    if not _distinct(dst, row_bytes):
        _refuse("a state cannot be written twice in one call")
    parent = parent.contiguous()
    n = len(states)
    numbers = array("q", (*src, *dst, *row_bytes, *src_batch, *src_beam, *dst_batch, *dst_beam))      # seven arrays of n entries
    at = numbers.buffer_info()[0]
    with _on(device):
        B.ols_beam_reorder(n, *range(at, at + 7 * 8 * n, 8 * n), batch, have, beams, parent.data_ptr(), _stream(device))
    return outs


# ---- products in 8-bit integers -----------------------------------------------------------------------------------
Int8Rows = namedtuple("Int8Rows", "q scale")
Int8Weight = namedtuple("Int8Weight", "q scale")


_NO_MATRIX = B.ols_matrix(None, 0, 0)


def _padded(n):
    return -(-n // 16) * 16          # rows that begin on 16 bytes


def _scale(t, m, n, name):
    """Address and workers' stride of fp32 scales [n] or [m][n]."""
    shape = t.shape
    if t.dtype != torch.float32 or not (shape == (n,) or shape == (m, n)) or not t.is_contiguous():
        _refuse("%s must be contiguous float32 of shape %s, got %s of shape %s", name, (m, n), t.dtype, tuple(shape))
    return t.data_ptr(), (n if len(shape) == 2 and m > 1 else 0)


def _act_code(act):
    if act not in _ACT:
        _refuse("unknown activation %r: one of %s", act, ", ".join(_ACT))
    return _ACT[act]


def quantize_rows(x, up=None, act="silu"):
    """Rows of x, or of act(x) * up, in 8 bits: q = x / scale to the nearest whole number, scale = max |row| / 127.

    x, up: fp32 or bf16 [rows, width] or [m, rows, width].  Returns Int8Rows(q, scale) for int8_matmul: q int8 of x's shape, scale fp32 of
    x.shape[:-1].  A row with a NaN or an infinity has q 0 and a scale of NaN."""
    device = _on_gpu(x, up)
    if x.dim() not in (2, 3):
        _refuse("x is [rows, width] or [m, rows, width], got %d axes", x.dim())
    m, (rows, width) = (x.shape[0] if x.dim() == 3 else 1), x.shape[-2:]
    if up is not None and (up.shape != x.shape or up.dtype != x.dtype):
        _refuse("up must be of x's shape and type")
    mx, mu = _matrix(x, m, (rows, width), "x"), None if up is None else _matrix(up, m, (rows, width), "up")
    with _on(device):
        pitch = _padded(width)
        q = torch.empty(*x.shape[:-1], pitch, dtype=torch.int8, device=device)[..., :width]
        scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=device)
        B.ols_quantize_rows(m, rows, width, mx, mu, _act_code(act), _dtype(x, "x"), q.data_ptr(), pitch, rows * pitch, scale.data_ptr(), rows, _stream(device))
    return Int8Rows(q, scale)


def quantize_weight(w):
    """A weight [width, out] or [m, width, out] in 8 bits with a scale for each column, laid out once for int8_matmul.

    Returns Int8Weight(q, scale): q int8 [out, width] or [m, out, width], scale fp32 [out] or [m, out]."""
    device = _on_gpu(w)
    if w.dim() not in (2, 3):
        _refuse("a weight is [width, out] or [m, width, out], got %d axes", w.dim())
    m, (width, out) = (w.shape[0] if w.dim() == 3 else 1), w.shape[-2:]
    mw = _matrix(w, m, (width, out), "weight")
    nbytes = B.ols_quantize_weight_workspace_bytes(m, width, out)
    with _on(device):
        ws = _workspace(nbytes, device)
        pitch = _padded(width)
        q = torch.empty(*w.shape[:-2], out, pitch, dtype=torch.int8, device=device)[..., :width]
        scale = torch.empty(*w.shape[:-2], out, dtype=torch.float32, device=device)
        B.ols_quantize_weight(m, width, out, mw, _dtype(w, "a weight"), q.data_ptr(), pitch, out * pitch, scale.data_ptr(), out, _ptr(ws), nbytes, _stream(device))
    return Int8Weight(q, scale)


def int8_matmul(x, weight, up=None, act="silu", out=None, dtype=None):
    """y = x w in 8-bit integers: rows of x with a scale each, channels of w with a scale each, exact integer sums.

    x: fp32 or bf16 [rows, width] or [m, rows, width], quantised on the way, or what quantize_rows returned.  With `up` (of x's shape and type)
    the product is that of act(x) * up: the second one of a gated block, for a = x and b = up.  weight: Int8Weight, from quantize_weight or of any int8
    q [out, width] or [m, out, width]; rows that do not begin on 16 bytes are copied first in every call of more than 32 rows.  y is [rows, out],
    with the workers' axis if anything has one, of `dtype` (x's by default, bfloat16 for Int8Rows) or in `out`, which may lie on x or up where these are not Int8Rows.  width < 2^17."""
    given = isinstance(x, Int8Rows)
    xq, (wq, w_scale) = (x.q if given else x), weight
    device = _on_gpu(xq, wq, w_scale, up, out, *((x.scale,) if given else ()))
    if wq.dtype != torch.int8 or (given and xq.dtype != torch.int8):
        _refuse("quantised tensors must be int8")
    x_shape, w_shape = xq.shape, wq.shape
    if len(x_shape) not in (2, 3) or len(w_shape) not in (2, 3):
        _refuse("x is [rows, width] or [m, rows, width], a quantised weight [out, width] or [m, out, width]")
    workers = len(x_shape) == 3 or len(w_shape) == 3
    m = x_shape[0] if len(x_shape) == 3 else w_shape[0] if workers else 1
    rows, width, channels = x_shape[-2], x_shape[-1], w_shape[-2]
    code = B.OLS_I8 if given else _dtype(xq, "x")
    dtype = dtype or (out.dtype if out is not None else torch.bfloat16 if given else xq.dtype)
    mx, mw, mu = _matrix(xq, m, (rows, width), "x"), _matrix(wq, m, (channels, width), "weight"), _NO_MATRIX
    if up is not None:
        if given or up.dtype != xq.dtype:
            _refuse("up must be of x's type, which is not quantised yet")
        mu = _matrix(up, m, (rows, width), "up")
    xs = _scale(x.scale, m, rows, "the rows' scales") if given else (None, 0)
    ws = _scale(w_scale, m, channels, "the channels' scales")
    shape = (m, rows, channels) if workers else (rows, channels)
    with _on(device):
        if out is None:
            out = torch.empty(*shape, dtype=dtype, device=device)
        elif out.shape != shape or out.dtype != dtype:
            _refuse("out must be %s of shape %s", dtype, shape)
        f = B.ols_int8(m, code, _act_code(act), _dtype(dtype, "dtype"), rows, width, channels, mx, mu, mw, _matrix(out, m, (rows, channels), "out"), *xs, *ws)
        f.ws_bytes = B.ols_int8_workspace_bytes(f)
        space = _workspace(f.ws_bytes, device)
        f.ws = _ptr(space)
        B.ols_int8_matmul(f, _stream(device))
    return out
