"""Sizes at which a call of the feed-forward block would ask for more threads than a launch has, on the host: refused before anything is
launched."""
import pytest

from paper_2002_09539_amd import binding as B

A = 0x7F0000000000      # stand-in for device addresses; never dereferenced
BIG = 1 << 60


def block(groups, rows, width, hidden, out, dtype):
    f = B.ols_ffn()
    f.groups, f.act, f.dtype, f.weight_dtype, f.grad_dtype = groups, B.OLS_ACT_SILU, dtype, dtype, dtype
    f.rows, f.width, f.hidden, f.out = rows, width, hidden, out
    shapes = dict(x=(rows, width), w_gate=(width, hidden), w_up=(width, hidden), w_down=(hidden, out), y=(rows, out), dy=(rows, out),
                  dx=(rows, width), g_gate=(width, hidden), g_up=(width, hidden), g_down=(hidden, out))
    for name, (r, c) in shapes.items():
        setattr(f, name, B.ols_matrix(A, c, r * c))
    f.saved, f.saved_bytes, f.ws, f.ws_bytes = A, BIG, A, BIG
    return f


# tiles are 128 rows by 64 columns of a and b, 128 by 128 of the other products
@pytest.mark.parametrize("groups,rows,width,hidden,out,dtype", [(4096, 9, 8, 1 << 18, 8, B.OLS_F32), (4096, 9, 8, 1 << 19, 8, B.OLS_BF16),
                                                                 (4096, 9, 8, 8, 1 << 20, B.OLS_F32), (2, 1 << 24, 8, 8, 1 << 14, B.OLS_F32)])
def test_more_tiles_than_a_launch_numbers(groups, rows, width, hidden, out, dtype):
    f = block(groups, rows, width, hidden, out, dtype)
    for call in (lambda: B.ols_gated_ffn_workspace_bytes(f, 0), lambda: B.ols_gated_ffn(f, None)):
        with pytest.raises(B.OlsError, match="tiles") as e:
            call()
        assert e.value.code == B.OLS_EINVAL


def test_many_tiles_that_a_launch_numbers():
    assert B.ols_gated_ffn_workspace_bytes(block(4096, 9, 8, 64 * 4095, 8, B.OLS_F32), 0) > 0      # 2^24 - 4096
    assert B.ols_gated_ffn_workspace_bytes(block(4096, 9, 8, 1 << 16, 8, B.OLS_F32), 0) > 0
    assert B.ols_gated_ffn_workspace_bytes(block(1, 1 << 24, 8, 8, 4096, B.OLS_BF16), 1) > 0
