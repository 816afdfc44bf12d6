"""Host logic of the operators of token models, which needs no GPU: every refusal of the C boundary comes before a launch,
with a message, and workspace sizes follow the shapes."""
import ctypes as C

import pytest

from paper_2002_09539_amd import binding as B

A = 0x7F0000000000      # 256-byte aligned stand-in for device addresses; never dereferenced
F32, BF16 = B.OLS_F32, B.OLS_BF16
BIG = 1 << 60


def refused(call, code=B.OLS_EINVAL, part=""):
    with pytest.raises(B.OlsError) as e:
        call()
    assert e.value.code == code and part in str(e.value), str(e.value)


# ---- embeddings ------------------------------------------------------------------------------------------------------
EMBED = dict(groups=2, tokens=7, vocab=11, width=5, ids=A, ids_group=7, table=A, dtype=F32, table_row=5, table_group=55, scale=1.0, out=A,
             out_dtype=F32, out_row=5, out_group=35, stream=None)


@pytest.mark.parametrize("change", [dict(groups=0), dict(groups=4097), dict(tokens=-1), dict(tokens=2 ** 24 + 1), dict(vocab=0), dict(vocab=2 ** 24 + 1),
                                    dict(width=0), dict(width=2 ** 20 + 1), dict(ids=None), dict(table=None), dict(out=None), dict(ids=A + 2),
                                    dict(table=A + 2), dict(table=A + 1, dtype=BF16), dict(dtype=2), dict(out_dtype=-1), dict(table_row=4),
                                    dict(out_row=4), dict(out_group=34), dict(ids_group=-1), dict(table_group=1 << 41)])
def test_embed_refuses(change):
    refused(lambda: B.ols_embed(*{**EMBED, **change}.values()), part="ols_embed")


EMBED_GRAD = dict(groups=2, tokens=7, vocab=11, width=5, ids=A, ids_group=7, d_out=A, dtype=F32, d_out_row=5, d_out_group=35, scale=1.0, grad=A,
                  grad_dtype=F32, grad_row=5, grad_group=55, accumulate=0, ws=A, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [dict(groups=0), dict(tokens=-1), dict(vocab=0), dict(width=0), dict(ids=None), dict(d_out=None), dict(grad=None),
                                    dict(grad=A + 2), dict(d_out_row=4), dict(grad_row=4), dict(grad_group=54), dict(grad_dtype=7), dict(ws=A + 16)])
def test_embed_grad_refuses(change):
    refused(lambda: B.ols_embed_grad(*{**EMBED_GRAD, **change}.values()), part="ols_embed_grad")


def test_embed_grad_workspace():
    need = B.ols_embed_grad_workspace_bytes(2, 7, 11, 5)
    assert 0 < need < 1 << 16
    for change in (dict(ws=None), dict(ws_bytes=need - 1)):
        refused(lambda: B.ols_embed_grad(*{**EMBED_GRAD, **change}.values()), B.OLS_ENOMEM, str(need))
    refused(lambda: B.ols_embed_grad_workspace_bytes(0, 1, 1, 1))
    # lists of ids and positions twice, and partial rows of an eighth of the input's elements
    big = B.ols_embed_grad_workspace_bytes(1, 1 << 20, 50000, 1024)
    assert (1 << 20) * (16 + 1024 / 8 * 4) <= big <= (1 << 20) * (16 + 1024 / 8 * 4) * 1.01 + (1 << 20)


# ---- log probabilities -------------------------------------------------------------------------------------------------
LOGPROBS = dict(rows=3, vocab=100, logits=A, dtype=F32, stride=100, targets=A, logprob=A, entropy=A, lse=A, stats=A, top=4, top_logprob=A, top_index=A,
                d_logprob=A, d_entropy=A, d_logits=A, d_stride=100, ws=A, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=2 ** 24 + 1), dict(logits=None), dict(logits=A + 2),
                                    dict(dtype=3), dict(stride=99), dict(targets=A + 2), dict(logprob=None), dict(entropy=None), dict(lse=None),
                                    dict(stats=None), dict(top=-1), dict(top=33), dict(vocab=3, stride=100), dict(top_logprob=None), dict(top_index=None),
                                    dict(top_index=A + 1), dict(d_logits=A + 2), dict(d_stride=99), dict(d_stride=101), dict(d_logprob=A + 2)])
def test_logprobs_refuse(change):
    refused(lambda: B.ols_token_logprobs(*{**LOGPROBS, **change}.values()), part="ols_token_logprobs")


LOGPROBS_GRAD = dict(rows=3, vocab=100, logits=A, dtype=F32, stride=100, targets=A, stats=A, entropy=A, d_logprob=A, d_entropy=A, d_logits=A + 4096,
                     d_stride=100, stream=None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(vocab=0), dict(logits=None), dict(stats=None), dict(entropy=None), dict(d_logits=None),
                                    dict(d_stride=99), dict(stats=A + 1), dict(dtype=9)])
def test_logprobs_grad_refuses(change):
    refused(lambda: B.ols_token_logprobs_grad(*{**LOGPROBS_GRAD, **change}.values()), part="ols_token_logprobs_grad")


def test_logprobs_workspace():
    bytes_of = B.ols_token_logprobs_workspace_bytes
    assert bytes_of(0, 100, F32, 4) == 0 and bytes_of(4096, 50000, BF16, 8) == 0      # a workgroup holds a row
    assert bytes_of(1, 1 << 17, F32, 0) % 12 == 0 and bytes_of(1, 1 << 17, F32, 0) > 12
    assert bytes_of(1000, 1 << 18, F32, 2) == 1000 * 4 * (12 + 16)                    # four parts of 65 536
    for bad in [(-1, 5, F32, 0), (1, 0, F32, 0), (1, 5, 8, 0), (1, 5, F32, 6), (1, 100, F32, 33)]:
        refused(lambda: bytes_of(*bad))
    need = bytes_of(1, 1 << 17, F32, 4)
    refused(lambda: B.ols_token_logprobs(*{**LOGPROBS, **dict(rows=1, vocab=1 << 17, stride=1 << 17, d_stride=1 << 17, ws_bytes=need - 1)}.values()),
            B.OLS_ENOMEM)


# ---- gated feed-forward block ----------------------------------------------------------------------------------------------
def block(**change):
    f = B.ols_ffn()
    f.groups, f.act, f.dtype, f.weight_dtype, f.grad_dtype = 2, B.OLS_ACT_SILU, BF16, BF16, F32
    f.rows, f.width, f.hidden, f.out = 40, 16, 32, 24
    shapes = dict(x=(40, 16), w_gate=(16, 32), w_up=(16, 32), w_down=(32, 24), y=(40, 24), dy=(40, 24), dx=(40, 16), g_gate=(16, 32), g_up=(16, 32),
                  g_down=(32, 24))
    for name, (r, c) in shapes.items():
        setattr(f, name, B.ols_matrix(A, c, r * c))
    f.saved, f.saved_bytes, f.ws, f.ws_bytes = A, BIG, A, BIG
    for name, value in change.items():
        at = f
        *path, last = name.split("__")
        for p in path:
            at = getattr(at, p)
        setattr(at, last, value)
    return f


BOTH = [dict(groups=0), dict(groups=4097), dict(act=3), dict(act=-1), dict(dtype=2), dict(weight_dtype=5), dict(grad_dtype=-2), dict(dtype=F32),
        dict(dtype=F32, weight_dtype=F32, grad_dtype=BF16), dict(rows=-1), dict(rows=2 ** 24 + 1), dict(width=0), dict(hidden=2 ** 20 + 1), dict(out=0),
        dict(x__dev=None), dict(x__dev=A + 1), dict(x__row=15), dict(w_gate__dev=None), dict(w_up__row=31), dict(w_down__dev=A + 1), dict(w_down__row=23),
        dict(x__group=-1), dict(saved=A + 64), dict(saved_bytes=16)]


@pytest.mark.parametrize("change", BOTH + [dict(y__dev=None), dict(y__row=23), dict(y__group=40 * 24 - 1)])
def test_block_refuses(change):
    refused(lambda: B.ols_gated_ffn(block(**change), None), part="ols_gated_ffn")


@pytest.mark.parametrize("change", BOTH + [dict(dy__dev=None), dict(dy__row=1), dict(dx__row=3), dict(dx__group=1), dict(g_gate__group=511),
                                           dict(g_up__dev=A + 2), dict(g_down__row=23), dict(saved=None)])
def test_block_grad_refuses(change):
    refused(lambda: B.ols_gated_ffn_grad(block(**change), None), part="ols_gated_ffn_grad")


def test_block_workspace():
    f = block()
    saved = B.ols_gated_ffn_saved_bytes(f)
    assert saved >= 2 * 40 * 32 * (4 + 4 + 2)                    # a, b and h
    packed = B.ols_gated_ffn_workspace_bytes(block(x__dev=A + 2), 0) - B.ols_gated_ffn_workspace_bytes(f, 0)
    assert 2 * 40 * 16 * 2 <= packed <= 2 * 40 * 16 * 2 + 256     # x laid out; the others are read where they lie
    for grad, call in ((0, B.ols_gated_ffn), (1, B.ols_gated_ffn_grad)):
        need = B.ols_gated_ffn_workspace_bytes(f, grad)
        if need:
            refused(lambda: call(block(ws_bytes=need - 1), None), B.OLS_ENOMEM)
            refused(lambda: call(block(ws=None), None), B.OLS_ENOMEM)
    few = block(rows=3, saved=None)
    assert 0 < B.ols_gated_ffn_workspace_bytes(few, 0) < 1 << 20
    lib = B.load()
    assert lib.ols_gated_ffn(None, None) == B.OLS_EINVAL and lib.ols_gated_ffn_saved_bytes(None) == B.OLS_EINVAL


# ---- clipping ----------------------------------------------------------------------------------------------------------
def clip(n=3, inputs=(A, A, A), outputs=(A, A, A), numel=(4, 0, 9), group=(0, 0, 1), groups=2, dtype=F32, max_norm=1.0, norms=A, ws=A, ws_bytes=BIG):
    arr = lambda t, v: None if v is None else C.addressof(_keep(t, v))  # noqa: E731
    keep = []

    def _keep(t, v):
        a = (t * len(v))(*v)
        keep.append(a)
        return a
    B.ols_clip_gradients(n, arr(C.c_void_p, inputs), arr(C.c_void_p, outputs), arr(C.c_int64, numel), arr(C.c_int32, group), groups, dtype, max_norm,
                         norms, ws, ws_bytes, None)


@pytest.mark.parametrize("change", [dict(n=-1), dict(inputs=None), dict(numel=None), dict(groups=0), dict(groups=4097), dict(group=None), dict(dtype=4),
                                    dict(group=(0, 1, 0)), dict(group=(0, 0, 2)), dict(group=(-1, 0, 0)), dict(numel=(4, -1, 9)), dict(numel=(4, 1 << 41, 9)),
                                    dict(inputs=(A, A, None)), dict(outputs=(None, A, A)), dict(inputs=(A + 2, A, A)), dict(outputs=(A, A, A + 1)),
                                    dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norms=None), dict(norms=A + 2), dict(ws=A + 8)])
def test_clipping_refuses(change):
    refused(lambda: clip(**change), part="ols_clip_gradients")


def test_clipping_workspace():
    def need(numel, group, groups):
        n = (C.c_int64 * len(numel))(*numel)
        g = (C.c_int32 * len(group))(*group)
        return B.ols_clip_workspace_bytes(len(numel), C.addressof(n), C.addressof(g), groups)
    assert need([4, 0, 9], [0, 0, 1], 2) == 16 and need([16384, 16385], [0, 0], 1) == 24
    assert need([1 << 30], [0], 1) <= 8 * 2048 + 8
    refused(lambda: clip(ws_bytes=8), B.OLS_ENOMEM)
    refused(lambda: need([1, 1], [1, 0], 2))


def test_parameter_buffer_needs_a_bound_handle():
    h = B.ols_create(2, 100, 2, 0.5, 0.1, 0.0)
    refused(lambda: B.ols_params_buffer(h), B.OLS_ESTATE)
    B.ols_destroy(h)


def test_the_tensor_functions_refuse_the_cpu():
    import torch
    from paper_2002_09539_amd import operators as ops
    z, t = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32)
    w = torch.zeros(8, 8)
    for call in [lambda: ops.embed(w, t), lambda: ops.embed_grad(t, z, 5), lambda: ops.token_logprobs(z, t), lambda: ops.token_logprobs_with_grad(z, t, z[:, 0]),
                 lambda: ops.gated_ffn(z, w, w, w), lambda: ops.clip_grad_norm([z], 1.0), lambda: ops.grad_norm([z])]:
        refused(call, part="GPU")
