"""The gated feed-forward block, forward and backward, against 64 bits.

Tolerances, per tensor as the 2-norm of the difference over the 2-norm of the result (and a bound on single entries).
fp32: every product is good to 2^-23.9, sums of up to 3000 terms are rounded 6 / 16 times a term by 2^-24 of the running sum
(random signs: about sqrt(3000) 2^-24 of the terms' root mean square at the very worst, 3e-6 of the result), and a gradient
passes three such products: 1e-5.  bf16: a rounding to nearest is 2^-9 / sqrt(3) = 1.13e-3 in the root mean square; y rounds h and
itself, da and db carry the roundings of a, b and their own, their products another two and the result's: five independent ones
at most, 2.6e-3.  1e-2 in all, single entries 12 times that of the root mean square."""
import math

import pytest
import torch

from paper_2002_09539_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 1e-5, BF16: 1e-2}
NAMES = ("y", "dx", "dw_gate", "dw_up", "dw_down")


def _ops():
    from paper_2002_09539_amd import operators
    return operators


def _act(name, a):
    if name == "silu":
        return a * torch.sigmoid(a)
    if name == "gelu":
        return 0.5 * a * torch.erfc(-a / math.sqrt(2))
    return a.clamp(min=0)


def _slope(name, a):
    if name == "silu":
        s = torch.sigmoid(a)
        return s + a * s * (1 - s)
    if name == "gelu":
        return 0.5 * torch.erfc(-a / math.sqrt(2)) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    return (a > 0).double()


def _want(x, wg, wu, wd, act, dy=None):
    """Of one worker, in 64 bits, from the formulas."""
    x, wg, wu, wd = (t.double().cpu() for t in (x, wg, wu, wd))
    a, b = x @ wg, x @ wu
    f = _act(act, a)
    h = f * b
    if dy is None:
        return (h @ wd,)
    dy = dy.double().cpu()
    dh = dy @ wd.T
    da, db = dh * b * _slope(act, a), dh * f
    return h @ wd, da @ wg.T + db @ wu.T, x.T @ da, x.T @ db, h.T @ dy


def _near(got, want, tol, name):
    got = got.double().cpu()
    assert got.shape == want.shape, name
    norm = float(want.norm())
    if want.numel() == 0 or norm == 0.0:
        assert float(got.norm()) == 0.0 if want.numel() else True, name
        return
    off = got - want
    assert float(off.norm()) <= tol * norm, (name, float(off.norm()) / norm)
    assert float(off.abs().max()) <= 12 * tol * max(norm / math.sqrt(want.numel()), float(want.abs().max())), name


def _inputs(seed, m, rows, width, hidden, out, dtype, wdtype=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std  # noqa: E731
    wt = wdtype or dtype
    x, dy = r(m, rows, width).to(dtype), r(m, rows, out).to(dtype)
    return x, r(m, width, hidden, std=width ** -0.5).to(wt), r(m, width, hidden, std=width ** -0.5).to(wt), r(m, hidden, out, std=hidden ** -0.5).to(wt), dy


def _check(x, wg, wu, wd, dy, act, grad_dtype=None):
    m = x.shape[0]
    y, saved = _ops().gated_ffn(x, wg, wu, wd, act, save=True)
    plain = _ops().gated_ffn(x, wg, wu, wd, act)
    grads = _ops().gated_ffn_grad(dy, x, wg, wu, wd, saved, act, grad_dtype=grad_dtype)
    tol = TOL[x.dtype]
    for w in range(m):
        pick = lambda t: t[w] if t.dim() == 3 else t  # noqa: E731
        want = _want(pick(x), pick(wg), pick(wu), pick(wd), act, pick(dy))
        for name, got, ref in zip(NAMES, (y, *grads), want):
            _near(got[w], ref, tol, name)
        _near(plain[w], want[0], tol, "y without saving")
    assert all(g.dtype == (grad_dtype or wg.dtype) for g in grads[1:]) and grads.x.dtype == x.dtype
    again = _ops().gated_ffn_grad(dy, x, wg, wu, wd, saved, act, grad_dtype=grad_dtype)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


# single rows; a vector and one more; tiles of 128 and 256 hung over; a contraction cut into ranges; large tiles
SHAPES = [(1, 1, 1, 1, 1), (2, 3, 5, 7, 3), (1, 8, 64, 128, 72), (1, 9, 65, 130, 70), (3, 130, 72, 264, 40), (1, 257, 129, 131, 257), (2, 64, 1024, 512, 1000),
          (1, 1000, 300, 517, 131), (1, 2048, 256, 2560, 264)]


@pytest.mark.parametrize("m,rows,width,hidden,out", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_block(m, rows, width, hidden, out, dtype):
    act = ("silu", "gelu", "relu")[(rows + width) % 3]
    _check(*_inputs(rows, m, rows, width, hidden, out, dtype), act)


def test_large_tiles_in_every_product():
    _check(*_inputs(3, 1, 4096, 2560, 2568, 2600, BF16), "silu")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_activations(act, dtype):
    x, wg, wu, wd, dy = _inputs(11, 1, 70, 48, 96, 32, dtype)
    _check(x * 4, wg, wu, wd, dy, act)           # pre-activations of up to 16 either way


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8, 9, 33])
@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_few_rows(rows, dtype, wdtype):
    for width, hidden, out in [(2048, 640, 1032), (77, 2100, 3)]:
        x, wg, wu, wd, _ = _inputs(rows, 2, rows, width, hidden, out, dtype, wdtype)
        y = _ops().gated_ffn(x, wg, wu, wd, "silu")
        for w in range(2):
            _near(y[w], _want(x[w], wg[w], wu[w], wd[w], "silu")[0], TOL[dtype], "y")


@pytest.mark.parametrize("grad_dtype", [F32, BF16])
def test_master_weights(grad_dtype):
    """A bf16 block on fp32 weights that lie in parameter rows, its gradients in gradient rows."""
    m, rows, width, hidden, out = 2, 140, 40, 96, 24
    sizes = [width * hidden, width * hidden, hidden * out]
    ld = 4 + sum(sizes) + 60
    p = torch.randn(m, ld, device="cuda") * 0.2
    g = torch.zeros(m, ld, device="cuda", dtype=grad_dtype)
    shapes = [(width, hidden), (width, hidden), (hidden, out)]
    offs = [4, 4 + sizes[0], 4 + sizes[0] + sizes[1]]
    cut = lambda t: [t[:, o: o + s].unflatten(1, sh) for o, s, sh in zip(offs, sizes, shapes)]  # noqa: E731
    weights, grads = cut(p), cut(g)
    x, dy = torch.randn(m, rows, width, device="cuda").to(BF16), torch.randn(m, rows, out, device="cuda").to(BF16)
    y, saved = _ops().gated_ffn(x, *weights, save=True)
    got = _ops().gated_ffn_grad(dy, x, *weights, saved, out=_ops().FfnGrads(None, *grads))
    assert got.w_down is grads[2]
    for w in range(m):
        want = _want(x[w], *(t[w].to(BF16) for t in weights), "silu", dy[w])
        for name, have, ref in zip(NAMES, (y[w], got.x[w], *(t[w] for t in grads)), want):
            _near(have, ref, TOL[BF16], name)
    assert float(g[:, :4].abs().sum()) == 0.0 and float(g[:, 4 + sum(sizes):].abs().sum()) == 0.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_inputs_and_strides(dtype):
    """Workers that share x, or the weights; rows that lie apart and start anywhere."""
    m, rows, width, hidden, out = 3, 50, 24, 40, 16
    x, wg, wu, wd, dy = _inputs(2, m, rows, width, hidden, out, dtype)
    _check_pair = _ops().gated_ffn(x[0], wg, wu, wd)
    for w in range(m):
        _near(_check_pair[w], _want(x[0], wg[w], wu[w], wd[w], "silu")[0], TOL[dtype], "y")
    _check(x, wg[0], wu[0], wd[0], dy, "gelu")
    wide = torch.randn(m, rows, width + 9, device="cuda").to(dtype)[:, :, 1: 1 + width]
    far = torch.randn(m, width, hidden + 16, device="cuda").to(dtype)[:, :, 8: 8 + hidden] * 0.2
    _check(wide, far, wu, wd, dy, "silu")
    odd = (torch.randn(m * width * hidden + 1, device="cuda") * 0.2).to(dtype)[1:].view(m, width, hidden)
    _check(wide, odd, odd, wd, dy, "silu")


def test_some_gradients_only():
    ops = _ops()
    x, wg, wu, wd, dy = _inputs(4, 1, 100, 32, 64, 48, BF16)
    y, saved = ops.gated_ffn(x, wg, wu, wd, save=True)
    full = ops.gated_ffn_grad(dy, x, wg, wu, wd, saved)
    part = ops.gated_ffn_grad(dy, x, wg, wu, wd, saved, need_x=False)
    assert part.x is None and all(torch.equal(a, b) for a, b in zip(full[1:], part[1:]))


def test_no_rows():
    ops = _ops()
    x, wg, wu, wd, dy = _inputs(4, 2, 0, 32, 64, 48, BF16)
    y, saved = ops.gated_ffn(x, wg, wu, wd, save=True)
    g = ops.gated_ffn_grad(dy, x, wg, wu, wd, saved, grad_dtype=F32)
    assert y.shape == (2, 0, 48) and g.x.shape == (2, 0, 32)
    assert all(float(t.abs().max()) == 0.0 for t in g[1:])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nans_stay_in_their_rows(dtype):
    x, wg, wu, wd, dy = _inputs(8, 1, 140, 65, 130, 70, dtype)
    clean = _ops().gated_ffn(x, wg, wu, wd, "relu")
    x[0, 3, 7], x[0, 139, 64] = math.nan, math.inf
    y = _ops().gated_ffn(x, wg, wu, wd, "relu")
    keep = [i for i in range(140) if i not in (3, 139)]
    assert torch.equal(y[:, keep], clean[:, keep])
    assert torch.isnan(y[0, 3]).all() and not torch.isfinite(y[0, 139]).any()
    few = _ops().gated_ffn(x[:, 137:], wg, wu, wd, "relu")
    assert torch.isfinite(few[:, :2]).all() and not torch.isfinite(few[:, 2]).any()


def test_fp32_sums_of_infinities():
    """a = inf in one column keeps its sign through the three planes; the other column never meets it."""
    x = torch.zeros(1, 130, 4, device="cuda")
    x[0, :, 0] = math.inf
    x[0, :, 1] = 1.0
    wg = torch.zeros(1, 4, 8, device="cuda")
    wg[0, 0, :] = 0.37
    wu = torch.zeros(1, 4, 8, device="cuda")
    wu[0, 0, :] = -0.11
    wd = torch.full((1, 8, 2), 0.3, device="cuda")
    y = _ops().gated_ffn(x, wg, wu, wd, "relu")
    assert (y == -math.inf).all()


def test_gradient_against_differences():
    """Central differences, in 64 bits, of the formula's y; the loss is sum(dy y)."""
    x, wg, wu, wd, dy = _inputs(21, 1, 5, 6, 7, 4, F32)
    _, saved = _ops().gated_ffn(x, wg, wu, wd, "gelu", save=True)
    grads = _ops().gated_ffn_grad(dy, x, wg, wu, wd, saved, "gelu")
    args = [t[0].double().cpu() for t in (x, wg, wu, wd)]
    loss = lambda a: float((_want(*a, "gelu")[0] * dy[0].double().cpu()).sum())  # noqa: E731
    for k in range(4):
        for at in [(0, 0), (3, 2), (4, 3)]:
            up, down = [t.clone() for t in args], [t.clone() for t in args]
            up[k][at] += 1e-5
            down[k][at] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - float(grads[k][0][at])) <= 2e-5


def test_in_a_graph():
    ops = _ops()
    x, wg, wu, wd, dy = _inputs(5, 1, 200, 64, 128, 64, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        y, saved = ops.gated_ffn(x, wg, wu, wd, save=True)
        return (y, *ops.gated_ffn_grad(dy, x, wg, wu, wd, saved))

    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    for _ in range(3):
        x.mul_(-0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_refusals():
    ops = _ops()
    x, wg, wu, wd, dy = _inputs(1, 1, 4, 8, 16, 8, BF16)
    y, saved = ops.gated_ffn(x, wg, wu, wd, save=True)
    for call in [lambda: ops.gated_ffn(x, wg, wu, wd, "tanh"), lambda: ops.gated_ffn(x.half(), wg, wu, wd), lambda: ops.gated_ffn(x, wg, wu.float(), wd),
                 lambda: ops.gated_ffn(x.float(), wg, wu, wd), lambda: ops.gated_ffn(x, wg, wu[:, :, :8], wd), lambda: ops.gated_ffn(x, wg, wu, wg),
                 lambda: ops.gated_ffn(x[:, :, :4], wg, wu, wd), lambda: ops.gated_ffn(x.cpu(), wg, wu, wd), lambda: ops.gated_ffn(x, wg.transpose(1, 2), wu, wd),
                 lambda: ops.gated_ffn(x, wg, wu, wd, out=torch.zeros(1, 4, 8, device="cuda")), lambda: ops.gated_ffn_grad(dy.float(), x, wg, wu, wd, saved),
                 lambda: ops.gated_ffn_grad(dy, x, wg, wu, wd, saved[:256]), lambda: ops.gated_ffn_grad(dy, x, wg, wu, wd, saved, grad_dtype=torch.float16),
                 lambda: ops.gated_ffn_grad(dy[:, :2], x, wg, wu, wd, saved)]:
        with pytest.raises(B.OlsError):
            call()
