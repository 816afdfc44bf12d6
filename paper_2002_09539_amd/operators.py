"""Operators of token models on torch tensors: embedding lookup, gated feed-forward block, log probabilities, clipping.

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
    return _SAME if index == torch.cuda.current_device() else torch.cuda.device(index)


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
    have = tuple(t.shape)
    if have == shape and (m == 1 or name in _SHARED):
        t = t.unsqueeze(0)
    elif have != (m, *shape):
        _refuse("%s must be of shape %s, got %s", name, (m, *shape), have)
    group, row = _rows(t, name)
    return B.ols_matrix(t.data_ptr(), row, group)


def _saved(t):
    """Address and bytes of what a forward call left."""
    if t.dtype != torch.uint8 or t.dim() != 1 or not t.is_contiguous():
        _refuse("saved must be what gated_ffn(..., save=True) returned")
    return (t.data_ptr() if t.numel() else None), t.numel()


_SHARED = ("x", "w_gate", "w_up", "w_down", "dy")    # inputs that may come without a worker axis


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
    if t.dim() < 1 or t.shape[-1] < 1:
        _refuse("%s must have a last axis of tokens, got shape %s", name, tuple(t.shape))
    vocab = t.shape[-1]
    if t.dim() == 2 and (t.stride(1) == 1 or vocab == 1):
        return t, t.shape[0], t.stride(0) if t.shape[0] > 1 else vocab     # rows that overlap are refused by the boundary
    if not t.is_contiguous():
        _refuse("%s must be contiguous, or two-dimensional with contiguous rows", name)
    return t, t.numel() // vocab, vocab


def _per_row(t, shape, dtype, name):
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        _refuse("%s must be %s of shape %s, got %s of shape %s", name, dtype, tuple(shape), t.dtype, tuple(t.shape))
    return t.contiguous()


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
