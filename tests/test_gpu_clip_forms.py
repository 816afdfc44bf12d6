"""Clipping of very many tensors, of extreme limits, and tensors that are not to be clipped twice.

Tolerances as of the operator's own tests: a norm is the correctly rounded fp32 of a sum in 64 bits (2^-23), an element an fp32 product
with a coefficient rounded once (2^-22)."""
import ctypes as C

import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _many(sizes, groups):
    """Host arrays of a call over tensors that lie in one buffer, each on a line of its own."""
    pitch = 64
    assert max(sizes) <= pitch
    n = len(sizes)
    x, out = torch.randn(n, pitch, device="cuda"), torch.full((n, pitch), 7.0, device="cuda")
    at = lambda t: (C.c_void_p * n)(*range(t.data_ptr(), t.data_ptr() + n * pitch * 4, pitch * 4))  # noqa: E731
    arrays = [at(x), at(out), (C.c_int64 * n)(*sizes), (C.c_int32 * n)(*groups)]
    addresses = [C.addressof(a) for a in arrays]
    count = max(groups) + 1
    nbytes = B.ols_clip_workspace_bytes(n, addresses[2], addresses[3], count)
    ws, norms = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty(count, device="cuda")

    def call(max_norm):
        B.ols_clip_gradients(n, addresses[0], None if max_norm is None else addresses[1], addresses[2], addresses[3], count, B.OLS_F32, max_norm or 0.0,
                             norms.data_ptr(), ws.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
        return norms.clone()
    return call, x, out, arrays


# groups of fewer, of as many and of more chunks than the copies add up themselves, one behind the other
@pytest.mark.parametrize("counts", [[4096], [4097], [20_000], [10, 5000, 0, 4096, 9000, 1], [5000] * 3])
def test_groups_of_many_tensors(counts):
    r = torch.Generator().manual_seed(len(counts))
    sizes = torch.randint(0, 9, (sum(counts),), generator=r).tolist()
    sizes[0] = 5
    groups = [g for g, k in enumerate(counts) for _ in range(k)]
    call, x, out, _ = _many(sizes, groups)
    got = call(0.5)
    real = torch.arange(64, device="cuda")[None] < torch.tensor(sizes, device="cuda")[:, None]
    of = torch.tensor(groups, device="cuda")
    squares = torch.zeros(len(counts), dtype=torch.float64, device="cuda").index_add_(0, of, torch.where(real, x.double(), 0.0).square().sum(1))
    want = squares.sqrt()
    assert ((got.double() - want).abs() <= 2.0 ** -23 * want).all()
    scale = torch.where(want > 0.5, 0.5 / want, 1.0)[of][:, None]
    assert ((out.double() - x.double() * scale).abs()[real] <= 2.0 ** -22 * (x.double() * scale).abs()[real]).all()
    assert (out[~real] == 7.0).all()
    assert torch.equal(call(None), got)


def test_many_tensors_are_clipped_in_about_the_time_of_their_norm():
    """Where every workgroup of the copies adds up all tensors' sums, the time grows with the square of their number."""
    n = 50_000
    call, _, _, _ = _many([8] * n, [0] * n)

    def least(max_norm):
        call(max_norm)
        times = []
        for _ in range(3):
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            torch.cuda.synchronize()
            a.record()
            call(max_norm)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    norm, clip = least(None), least(1.0)
    print("%d tensors: norm %.2f ms, clipping %.2f ms" % (n, norm, clip))
    assert clip <= 5 * norm


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value,max_norm", [(1e36, 1e-3), (1e38, 1.0), (3e38, 1e-6), (1e15, 1e-30), (1e30, 1e-12), (1e-30, 1e-36)])
def test_factors_below_the_normal_numbers(dtype, value, max_norm):
    """max_norm / norm may be far below the least normal fp32 where gradients are huge or the limit is tiny; the results are not."""
    x = (torch.rand(100_000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * value).to(dtype)
    norm = float(x.double().square().sum().sqrt())
    want = x.double() * (max_norm / norm)
    big = want.abs() >= 2.0 ** -110                      # where the result is normal by a margin
    out = torch.empty_like(x)
    got = _ops().clip_grad_norm([x], max_norm, out=[out])
    assert norm > 3.4e38 or abs(float(got[0]) - norm) <= 2.0 ** -23 * norm
    assert int(big.sum()) > 90_000 or value == 1e-30 or max_norm == 1e-30
    assert ((out.double() - want).abs()[big] <= (2.0 ** -22 if dtype == F32 else 2.0 ** -8) * want.abs()[big]).all()


def test_a_tensor_is_not_scaled_twice():
    ops = _ops()
    x, y, none = torch.ones(50, device="cuda"), torch.ones(7, device="cuda"), torch.zeros(0, device="cuda")
    for call in (lambda: ops.clip_grad_norm([x, y, x], 1.0), lambda: ops.clip_grad_norm([x, x.clone()], 1.0, out=[x, x]),
                 lambda: ops.clip_grad_norm([x, y, x], 1.0, groups=[1, 0, 0])):
        with pytest.raises(B.OlsError, match="twice"):
            call()
    assert (x == 1).all()
    assert abs(float(ops.grad_norm([x, x])[0]) - 10.0) <= 1e-6                      # to read it twice is no harm
    two = [torch.empty_like(x), torch.empty_like(x)]
    ops.clip_grad_norm([x, x], 1.0, out=two)
    assert torch.equal(two[0], two[1]) and ((two[0] - 0.1).abs() <= 1e-7).all()
    ops.clip_grad_norm([none, x[:0], x, none.clone()], 1.0)
    assert abs(float(x.norm()) - 1.0) <= 1e-6
