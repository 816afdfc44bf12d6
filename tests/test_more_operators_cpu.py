"""Host logic of distillation, beam search and the products in 8-bit integers, which needs no GPU: every refusal of the C boundary comes
before a launch, with a message, and workspace sizes follow the shapes."""
import ctypes as C
from array import array

import pytest

from paper_2002_09539_amd import binding as B

A = 0x7F0000000000      # 256-byte aligned stand-in for device addresses; never dereferenced
F32, BF16, I8 = B.OLS_F32, B.OLS_BF16, B.OLS_I8
BIG = 1 << 60


def refused(call, code=B.OLS_EINVAL, part=""):
    with pytest.raises(B.OlsError) as e:
        call()
    assert e.value.code == code and part in str(e.value), str(e.value)


def filled(struct, values, change):
    s = struct()
    for k, v in {**values, **change}.items():
        setattr(s, k, v)
    return s


# ---- distillation -----------------------------------------------------------------------------------------------------
DISTILL = dict(dtype=F32, k=4, rest=1, temperature=2.0, rows=3, vocab=100, logits=A, row_stride=100, top_value=A, top_index=A, targets=A, loss=A, logprob=A,
               stats=A, d_loss=A, d_logprob=A, d_logits=A, d_stride=100, ws=A, ws_bytes=BIG)
ANY = [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=2 ** 24 + 1), dict(k=0), dict(k=257), dict(temperature=0.0), dict(temperature=-1.0),
       dict(temperature=float("nan")), dict(temperature=2.0 ** 21), dict(dtype=2), dict(logits=None), dict(logits=A + 2), dict(logits=A + 1, dtype=BF16),
       dict(row_stride=99), dict(top_value=None), dict(top_index=None), dict(top_value=A + 2), dict(top_index=A + 1), dict(targets=A + 2), dict(stats=None),
       dict(stats=A + 2), dict(d_loss=A + 2), dict(d_logprob=A + 1), dict(d_logits=A + 2), dict(d_stride=99), dict(d_stride=101)]


@pytest.mark.parametrize("change", ANY + [dict(loss=None), dict(logprob=None), dict(loss=A + 2), dict(ws=A + 16, rows=1, vocab=1 << 17, row_stride=1 << 17, d_stride=1 << 17)])
def test_distill_refuses(change):
    refused(lambda: B.ols_distill_loss(filled(B.ols_distill, DISTILL, change), None), part="ols_distill_loss")


@pytest.mark.parametrize("change", ANY + [dict(d_logits=None)])
def test_distill_grad_refuses(change):
    refused(lambda: B.ols_distill_loss_grad(filled(B.ols_distill, DISTILL, change), None), part="ols_distill_loss_grad")


def test_distill_workspace_and_no_rows():
    bytes_of = B.ols_distill_workspace_bytes
    assert bytes_of(0, 100, F32, 4) == 0 and bytes_of(1, 1 << 24, BF16, 4) > 0 and 0 < bytes_of(4096, 50000, BF16, 64) < 4096 * 1024
    refused(lambda: bytes_of(-1, 100, F32, 4))
    refused(lambda: bytes_of(1, 0, F32, 4))
    refused(lambda: bytes_of(1, 10, I8, 4))
    refused(lambda: bytes_of(1, 10, F32, 0))
    refused(lambda: bytes_of(1, 10, F32, 257))
    need = bytes_of(1, 1 << 17, F32, 4)
    few = dict(rows=1, vocab=1 << 17, row_stride=1 << 17, d_stride=1 << 17)
    refused(lambda: B.ols_distill_loss(filled(B.ols_distill, DISTILL, dict(**few, ws_bytes=need - 1)), None), B.OLS_ENOMEM, str(need))
    refused(lambda: B.ols_distill_loss(filled(B.ols_distill, DISTILL, dict(**few, ws=None)), None), B.OLS_ENOMEM)
    B.ols_distill_loss(filled(B.ols_distill, DISTILL, dict(rows=0, logits=None, loss=None)), None)
    refused(lambda: B._check(B.load().ols_distill_loss(None, None)), part="null")


# ---- beam search ------------------------------------------------------------------------------------------------------
BEAM = dict(dtype=F32, in_beams=3, beams=4, eos=2, batch=2, vocab=100, logits=A, batch_stride=300, beam_stride=100, score=A, finished=A + 1, length=A,
            length_penalty=1.0, new_score=A, token=A, parent=A, new_length=A, new_finished=A + 3, ws=A, ws_bytes=BIG)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(in_beams=0), dict(in_beams=33), dict(beams=0), dict(beams=33), dict(batch=-1), dict(batch=65536), dict(vocab=0),
                                    dict(vocab=2 ** 24 + 1), dict(logits=None), dict(logits=A + 2), dict(batch_stride=-1), dict(beam_stride=1 << 41), dict(score=None),
                                    dict(score=A + 2), dict(length=A + 2), dict(length=None), dict(length=None, length_penalty=0.0), dict(length_penalty=17.0),
                                    dict(length_penalty=float("nan")), dict(new_score=None), dict(token=None), dict(parent=None), dict(new_finished=None),
                                    dict(new_score=A + 1), dict(token=A + 2), dict(parent=A + 3), dict(new_length=A + 1), dict(ws=A + 8)])
def test_beam_refuses(change):
    refused(lambda: B.ols_beam_select(filled(B.ols_beam, BEAM, change), None), part="ols_beam_select")


def test_beam_workspace():
    need = B.ols_beam_workspace_bytes(2, 3, 4, 100, F32)
    assert need >= 6 * (12 + 32)
    refused(lambda: B.ols_beam_select(filled(B.ols_beam, BEAM, dict(ws_bytes=need - 1)), None), B.OLS_ENOMEM, str(need))
    refused(lambda: B.ols_beam_workspace_bytes(2, 33, 4, 100, F32))
    assert B.ols_beam_workspace_bytes(0, 3, 4, 100, F32) == 0
    shared = dict(batch=65535, in_beams=32, vocab=1 << 20, batch_stride=0, beam_stride=0)          # one row of logits for all
    refused(lambda: B.ols_beam_workspace_bytes(65535, 32, 4, 1 << 20, F32), part="2^24 parts")
    refused(lambda: B.ols_beam_select(filled(B.ols_beam, BEAM, shared), None), part="2^24 parts")
    B.ols_beam_select(filled(B.ols_beam, BEAM, dict(batch=0, logits=None)), None)


REORDER = dict(src=A, dst=A + (1 << 20), row_bytes=40, src_batch=120, src_beam=40, dst_batch=160, dst_beam=40)


def reorder(n=1, batch=2, in_beams=3, beams=4, parent=A, null=False, **change):
    values = {**REORDER, **change}
    arrays = [array("Q" if k in ("src", "dst") else "q", [v] * max(1, n)) for k, v in values.items()]
    at = [None if null else a.buffer_info()[0] for a in arrays]
    B.ols_beam_reorder(n, *at, batch, in_beams, beams, parent, None)


@pytest.mark.parametrize("change", [dict(n=-1), dict(n=(1 << 20) + 1), dict(batch=-1), dict(batch=65536), dict(in_beams=0), dict(beams=33), dict(parent=None), dict(parent=A + 2),
                                    dict(null=True), dict(src=0), dict(dst=0), dict(row_bytes=-1), dict(src_batch=-1), dict(src_beam=1 << 41), dict(dst_beam=39),
                                    dict(dst_batch=159), dict(dst=A), dict(dst=A, beams=3), dict(dst=A + 8), dict(dst=A + 239)])
def test_reorder_refuses(change):
    refused(lambda: reorder(**change), part="ols_beam_reorder")


def test_reorder_of_nothing():
    reorder(n=0, parent=None)
    reorder(batch=0)
    reorder(row_bytes=0, src=0, dst=0)


# ---- products in 8 bits -----------------------------------------------------------------------------------------------
def matrix(dev=A, row=64, group=6400):
    return B.ols_matrix(dev, row, group)


INT8 = dict(groups=2, dtype=BF16, act=0, out_dtype=F32, rows=70, width=40, out=30, x=matrix(), up=matrix(None), w=matrix(), y=matrix(), x_scale=A, x_scale_group=70,
            w_scale=A, w_scale_group=30, ws=A, ws_bytes=BIG)


@pytest.mark.parametrize("change", [dict(groups=0), dict(groups=4097), dict(dtype=3), dict(out_dtype=2), dict(act=3), dict(rows=-1), dict(rows=2 ** 24 + 1), dict(width=0),
                                    dict(width=2 ** 17), dict(out=0), dict(out=2 ** 24 + 1), dict(rows=2 ** 24, out=2 ** 13, y=matrix(row=2 ** 13)), dict(rows=64, out=2 ** 24), dict(x=matrix(None)), dict(x=matrix(A + 1)),
                                    dict(x=matrix(row=39)), dict(x=matrix(group=-1)), dict(up=matrix(A + 1)), dict(up=matrix(row=39)), dict(w=matrix(None)), dict(w=matrix(row=39)),
                                    dict(w=matrix(group=1 << 41)), dict(w_scale=None), dict(w_scale=A + 2), dict(w_scale_group=-1), dict(y=matrix(None)), dict(y=matrix(A + 2)),
                                    dict(y=matrix(row=29)), dict(y=matrix(group=29)), dict(ws=A + 128), dict(dtype=I8, up=matrix()), dict(dtype=I8, x_scale=None),
                                    dict(dtype=I8, x_scale=A + 1), dict(dtype=I8, x=matrix(row=39))])
def test_int8_refuses(change):
    refused(lambda: B.ols_int8_matmul(filled(B.ols_int8, INT8, change), None), part="ols_int8_matmul")


def test_int8_workspace():
    f = filled(B.ols_int8, INT8, {})
    need = B.ols_int8_workspace_bytes(f)
    assert need >= 2 * 70 * 40
    refused(lambda: B.ols_int8_matmul(filled(B.ols_int8, INT8, dict(ws_bytes=need - 1)), None), B.OLS_ENOMEM, str(need))
    assert B.ols_int8_workspace_bytes(filled(B.ols_int8, INT8, dict(rows=0))) == 0
    refused(lambda: B.ols_int8_workspace_bytes(filled(B.ols_int8, INT8, dict(width=0))))
    B.ols_int8_matmul(filled(B.ols_int8, INT8, dict(rows=0, x=matrix(None), ws=None)), None)


QUANT = dict(groups=2, rows=5, width=40, x=matrix(), up=None, act=0, dtype=F32, q=A, q_row=48, q_group=240, scale=A, scale_group=5, stream=None)


@pytest.mark.parametrize("change", [dict(groups=0), dict(rows=-1), dict(width=0), dict(width=2 ** 17), dict(act=-1), dict(dtype=I8), dict(x=matrix(A + 2)), dict(x=matrix(row=39)),
                                    dict(up=matrix(A + 2)), dict(q=None), dict(q_row=39), dict(q_group=39), dict(scale=None), dict(scale=A + 2), dict(scale_group=4)])
def test_quantize_rows_refuses(change):
    refused(lambda: B.ols_quantize_rows(*{**QUANT, **change}.values()), part="ols_quantize_rows")


WEIGHT = dict(groups=2, width=40, out=30, w=matrix(), dtype=F32, q=A, q_row=48, q_group=48 * 30, scale=A, scale_group=30, ws=A, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [dict(groups=0), dict(width=0), dict(width=2 ** 17), dict(out=0), dict(out=2 ** 24 + 1), dict(dtype=I8), dict(w=matrix(A + 2)), dict(w=matrix(row=29)),
                                    dict(q=None), dict(q_row=39), dict(q_group=39), dict(scale=None), dict(scale_group=29), dict(ws=A + 4),
                                    dict(width=2 ** 16, out=2 ** 21, w=matrix(row=2 ** 21, group=0), q_row=2 ** 16, q_group=2 ** 38, scale_group=2 ** 21)])
def test_quantize_weight_refuses(change):
    refused(lambda: B.ols_quantize_weight(*{**WEIGHT, **change}.values()), part="ols_quantize_weight")


def test_quantize_weight_workspace():
    need = B.ols_quantize_weight_workspace_bytes(2, 40, 30)
    assert need >= 240
    refused(lambda: B.ols_quantize_weight(*{**WEIGHT, **dict(ws_bytes=need - 1)}.values()), B.OLS_ENOMEM, str(need))
    refused(lambda: B.ols_quantize_weight_workspace_bytes(2, 2 ** 17, 30))


def test_structures_are_those_of_the_header():
    """Sizes of the descriptors: every field has its place."""
    assert C.sizeof(B.ols_distill) == 4 * 4 + 8 * 2 + 8 * 2 + 8 * 9 + 8 * 3
    assert C.sizeof(B.ols_beam) == 4 * 4 + 8 * 2 + 8 * 3 + 8 * 3 + 8 + 8 * 6 + 8
    assert C.sizeof(B.ols_int8) == 4 * 4 + 8 * 3 + 24 * 4 + 8 * 6
