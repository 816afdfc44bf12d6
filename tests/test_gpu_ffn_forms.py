"""What the gated feed-forward block promises across its forms: calls of few and of more rows, with and without `saved`."""
import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2002_09539_amd import operators
    return operators


@pytest.mark.parametrize("rows", [1, 2, 4, 8, 9, 40])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("width,hidden,out", [(64, 40, 24), (300, 77, 9)])
def test_master_weights_are_rounded_whatever_the_rows(rows, save, width, hidden, out):
    """Weights a little above the middle between two bf16 numbers: rounded, each is 0.95 2^-8 larger, y (three of them) 1.1 %.  Of h and y at
    most two roundings of 2^-9 remain."""
    w = 1.0 + 1.05 * 2.0 ** -8
    x = torch.ones(rows, width, dtype=BF16, device="cuda")
    args = [torch.full(s, w * k, device="cuda") for s, k in (((width, hidden), 2.0 ** -6), ((width, hidden), 2.0 ** -6), ((hidden, out), 2.0 ** -4))]
    y = _ops().gated_ffn(x, *args, "relu", save=save)
    y = y[0] if save else y
    r = 1.0 + 2.0 ** -7
    assert torch.equal(args[0].to(BF16).float(), torch.full_like(args[0], r * 2.0 ** -6))
    want = (width * r * 2.0 ** -6) ** 2 * hidden * r * 2.0 ** -4
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want).all(), float(y[0, 0]) / want


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,rows,width,hidden", [(1, 3, 16, 24), (2, 40, 72, 136), (1, 300, 65, 50)])
def test_the_gradient_at_x_may_lie_on_x_or_on_dy(dtype, m, rows, width, hidden):
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-2] ** -0.5).to(dtype)  # noqa: E731
    x, dy = torch.randn(m, rows, width, generator=g, device="cuda").to(dtype), torch.randn(m, rows, width, generator=g, device="cuda").to(dtype)
    w = r(m, width, hidden), r(m, width, hidden), r(m, hidden, width)
    ops = _ops()
    _, saved = ops.gated_ffn(x, *w, save=True)
    want = ops.gated_ffn_grad(dy, x, *w, saved)
    for name in ("x", "dy"):
        xs, ds = x.clone(), dy.clone()
        got = ops.gated_ffn_grad(ds, xs, *w, saved, out=ops.FfnGrads(xs if name == "x" else ds, None, None, None))
        assert got.x is (xs if name == "x" else ds)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
    here = [t.clone() for t in w]            # the weights' gradients over the weights
    got = ops.gated_ffn_grad(dy, x, *here, saved, out=ops.FfnGrads(None, *here))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_saved_states_that_are_not_whole_are_refused():
    ops = _ops()
    x, w = torch.randn(20, 16, device="cuda"), [torch.randn(16, 16, device="cuda") for _ in range(3)]
    _, saved = ops.gated_ffn(x, *w, save=True)
    for t in (saved[:1].expand(saved.numel()), torch.zeros(2 * saved.numel(), dtype=torch.uint8, device="cuda")[::2], saved.float()):
        with pytest.raises(B.OlsError, match="saved"):
            ops.gated_ffn_grad(x, x, *w, t)


@pytest.mark.parametrize("rows", [1, 5, 60, 300])
def test_fp32_activations_far_below_zero(rows):
    """SiLU and its slope are small there but no less precise: an exponential, a sum, a division and a product, each rounded by 2^-24
    or a little more (2^-21 in all; the slope 2^-20, with two more products and a sum).  a = x w_gate and b = x w_up are exact."""
    a = torch.linspace(-80.0, -4.0, rows, device="cuda") if rows > 1 else torch.tensor([-61.3], device="cuda")
    x = torch.stack([a, torch.ones_like(a)], 1)
    wg, wu, wd = (torch.tensor(v, device="cuda") for v in ([[1.0], [0.0]], [[0.0], [1.0]], [[1.0]]))
    d = a.double()
    s = 1 / (1 + torch.exp(-d))
    want, slope = d * s, s + d * s * (1 - s)
    y, saved = _ops().gated_ffn(x, wg, wu, wd, save=True)
    for got in (y, _ops().gated_ffn(x, wg, wu, wd)):
        assert ((got[:, 0].double() - want).abs() <= 2.0 ** -21 * want.abs()).all()
    dx = _ops().gated_ffn_grad(torch.ones_like(y), x, wg, wu, wd, saved).x
    assert ((dx[:, 0].double() - slope).abs() <= 2.0 ** -20 * slope.abs()).all()
    assert ((dx[:, 1].double() - want).abs() <= 2.0 ** -21 * want.abs()).all()


@pytest.mark.parametrize("rows", [4, 40])
def test_fp32_silu_of_large_arguments(rows):
    """Where the exponential overflows or vanishes SiLU is its argument or nothing; of an infinite one it is that."""
    x = torch.ones(rows, 2, device="cuda")
    x[:4, 0] = torch.tensor([1e30, 300.0, 0.0, -300.0], device="cuda")
    wg, wu, wd = (torch.tensor(v, device="cuda") for v in ([[1.0], [0.0]], [[0.0], [1.0]], [[1.0]]))
    for y in (_ops().gated_ffn(x, wg, wu, wd), _ops().gated_ffn(x, wg, wu, wd, save=True)[0]):
        assert torch.equal(y[:4, 0], torch.tensor([1e30, 300.0, 0.0, 0.0], device="cuda"))
    one, far = torch.ones(1, 1, device="cuda"), torch.full((rows, 1), float("inf"), device="cuda")
    for y in (_ops().gated_ffn(far, one, one, one), _ops().gated_ffn(far, one, one, one, save=True)[0]):
        assert (y == float("inf")).all()
