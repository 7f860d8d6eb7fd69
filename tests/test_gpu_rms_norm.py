"""RMS norm with the residual's addition against its definition in float64.

Tolerances (relative in the 2-norm).  float32: one rounding per operation on a value (at most eight of 2^-24) and a sum whose roundings act on a common factor of the row:
16 * 2^-24; sums of gradients over rows: 64 * 2^-24 (as many additions in a chain).  bfloat16: the rounding of the result to 8 significant bits, 2^-8 at worst and
2^-8 / sqrt(3) times at most 0.86 (values between powers of two) < 2^-9 in the root mean square, with 1 / 8 on top for the float32 part.
8 bits: to the nearest of e4m3, half of its step, which is 2^-4 of the value (2^-10 for values below 2^-6), plus float32 roundings.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 16 * 2.0 ** -24
TOL = {torch.float32: F32, torch.bfloat16: 2.0 ** -9 * 1.125}
EPS = 1e-5


def close(got, want, tol, what):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    if want.numel():
        assert float((got - want).norm()) <= tol * float(want.norm()) + 1e-30, (what, float((got - want).norm() / want.norm()))
        rms = float(want.norm()) / math.sqrt(want.numel())
        assert float(((got - want).abs() - 8 * tol * want.abs().clamp(min=rms)).max()) <= 1e-30, (what, "element")


def make(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    t = lambda: (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)
    return dict(x=t(), residual=t(), weight=1 + 0.3 * torch.randn(cols, generator=g), dy=t(), dr=t())


def definition(x, weight, residual, dtype):
    r = (x.double() if residual is None else (x.float() + residual.float()).to(dtype).double()).requires_grad_(True)
    w = (torch.ones(x.shape[1]) if weight is None else weight).double().requires_grad_(True)
    rstd = 1 / torch.sqrt(r.pow(2).mean(1, keepdim=True) + EPS)
    return r, w, rstd, r * rstd * w


SIZES = [(1, 1), (3, 7), (5, 16), (33, 64), (9, 100), (130, 128), (17, 200), (7, 256), (4, 500), (66, 512), (5, 1000), (3, 1023), (6, 2048), (2, 3001), (3, 4096), (2, 8191), (2, 8192),
         (5000, 64), (3000, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("with_residual,with_weight", [(True, True), (False, True), (True, False)])
def test_forward_and_backward(rows, cols, dtype, with_residual, with_weight):
    from paper_2507_08637_amd import autograd
    p = make(rows, cols, dtype, rows + cols)
    g = {k: t.cuda() for k, t in p.items()}
    x = g["x"].requires_grad_(True)
    weight = g["weight"].requires_grad_(True) if with_weight else None
    residual = g["residual"].requires_grad_(True) if with_residual else None
    leaves = [t for t in (x, weight, residual) if t is not None]
    r64, w64, _, y64 = definition(p["x"], p["weight"] if with_weight else None, p["residual"] if with_residual else None, dtype)
    if with_residual:
        y, r = autograd.wersa_rms_norm(x, weight, residual, eps=EPS)
        assert torch.equal(r.detach().double().cpu(), r64.detach())
        grads = torch.autograd.grad((y, r), leaves, (g["dy"], g["dr"]))
        want_r, want_w = torch.autograd.grad((y64, r64 * 1), (r64, w64), (p["dy"].double(), p["dr"].double()))
        assert torch.equal(grads[0], grads[-1])
    else:
        y = autograd.wersa_rms_norm(x, weight, eps=EPS)
        grads = torch.autograd.grad(y, leaves, g["dy"])
        want_r, want_w = torch.autograd.grad(y64, (r64, w64), p["dy"].double())
    close(y, y64, TOL[dtype], "y")
    # dx is a difference of two terms: roundings of 2^-24 act on each, of a size that the difference may be far below (one column: it is nothing but eps)
    gy = (p["dy"].double() * w64.detach()) / torch.sqrt(r64.detach().pow(2).mean(1, keepdim=True) + EPS)
    err = (grads[0].double().cpu() - want_r).abs()
    row = gy.abs().amax(1, keepdim=True)
    result = 0.0 if dtype == torch.float32 else 2.0 ** -8
    assert (err <= result * want_r.abs() + 4 * F32 * (row * math.sqrt(cols) + want_r.abs()) + 1e-30).all()
    if with_weight:
        terms = (p["dy"].double() * r64.detach() / torch.sqrt(r64.detach().pow(2).mean(1, keepdim=True) + EPS)).norm(dim=0)
        assert ((grads[1].double().cpu() - want_w).abs() <= 64 * 2.0 ** -24 * (terms + want_w.abs()) + 1e-30).all()


def e4m3_step(v):
    """Distance of neighbouring e4m3 values at |v|."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("with_residual", [True, False])
def test_eight_bit(rows, cols, dtype, with_residual):
    from paper_2507_08637_amd import binding
    p = make(rows, cols, dtype, rows * 3 + cols)
    p["x"][rows // 2] = 0
    p["residual"][rows // 2] = 0
    g = {k: t.cuda() for k, t in p.items()}
    y, r, scales = binding.wersa_rms_norm_eight_bit(g["x"], g["weight"], residual=g["residual"] if with_residual else None, eps=EPS)
    r64, _, _, y64 = definition(p["x"], p["weight"], p["residual"] if with_residual else None, dtype)
    assert torch.equal(r.double().cpu(), r64.detach())
    most = y64.detach().abs().amax(1)
    close(scales, torch.where(most > 0, most / 448, torch.ones(()).double()), F32, "scales")
    assert scales[rows // 2] == 1 and (y[rows // 2].float() == 0).all()
    exact = y64.detach() * torch.where(most > 0, 448 / most, torch.ones(()).double())[:, None]
    err = (y.double().cpu() - exact).abs()
    assert (err <= e4m3_step(exact * (1 + 1e-6)) / 2 + F32 * exact.abs()).all()
    assert (y.float().abs().amax(1)[scales != 1] == 448).all()


def test_strided_rows_streams_and_not_a_number():
    from paper_2507_08637_amd import binding
    p = {k: t.cuda() for k, t in make(40, 96, torch.bfloat16).items()}
    wide = torch.zeros(40, 301, dtype=torch.bfloat16, device="cuda")
    x, res = wide[:, 1:97], wide[:, 150:246]
    x.copy_(p["x"])
    res.copy_(p["residual"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, r, _ = binding.wersa_rms_norm_forward(x, p["weight"], residual=res)
    side.synchronize()
    want, want_r, _ = binding.wersa_rms_norm_forward(p["x"], p["weight"], residual=p["residual"])
    assert torch.equal(y, want) and torch.equal(r, want_r)
    p["x"][3, 5], p["x"][7, 2] = float("nan"), float("inf")
    y, _, scales = binding.wersa_rms_norm_eight_bit(p["x"], p["weight"])
    z, _, _ = binding.wersa_rms_norm_forward(p["x"], p["weight"])
    fine = [i for i in range(40) if i not in (3, 7)]
    assert torch.isfinite(z[fine]).all() and z[3].isnan().all() and z[7, 2].isnan() and (z[7, :2] == 0).all()
    assert not y[fine].float().isnan().any() and y[3].float().isnan().all() and y[7, 2].float().isnan()


def test_no_rows():
    from paper_2507_08637_amd import autograd
    x = torch.empty(0, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    y = autograd.wersa_rms_norm(x, w)
    dx, dw = torch.autograd.grad(y.sum(), (x, w))
    assert y.shape == (0, 64) and dx.shape == (0, 64) and (dw == 0).all()


def test_leading_dimensions_and_unused_outputs():
    from paper_2507_08637_amd import autograd
    p = {k: t.cuda() for k, t in make(24, 64, torch.float32).items()}
    x, w, res = p["x"].view(2, 3, 4, 64).requires_grad_(True), p["weight"].requires_grad_(True), p["residual"].view(2, 3, 4, 64)
    y, r = autograd.wersa_rms_norm(x, w, residual=res)
    assert y.shape == x.shape and r.shape == x.shape
    (dx,) = torch.autograd.grad(r, x, p["dr"].view_as(r), retain_graph=True)
    assert torch.equal(dx.view(24, 64), p["dr"])
    one = torch.ones((), device="cuda")
    (dx,) = torch.autograd.grad(y, x, one.expand_as(y))
    (want,) = torch.autograd.grad(y_of := autograd.wersa_rms_norm(x, w, residual=res)[0], x, torch.ones_like(y))
    assert torch.equal(dx, want)


def test_more_rows_than_one_dimension_of_a_grid_has_threads_for():
    """2^29 rows of one column: 2^24 workgroups, 2^32 threads."""
    from paper_2507_08637_amd import binding
    rows = (1 << 29) + 5
    x = torch.full((rows, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    x[-1], x[-7], x[rows // 2] = -3.0, 0.0, -1.0
    y, _, _ = binding.wersa_rms_norm_forward(x, eps=0.0)
    y[-7] = 1
    assert (y[-1] == -1).all() and (y[rows // 2] == -1).all() and int((y == 1).sum()) == rows - 2
