"""Layer norm with the residual's addition against its definition in float64.

Tolerances.  m is a sum of cols values in float32, lane by lane and then over lanes: its roundings are at most 2^-24 of sum |r| / cols each, taken 16-fold for the chains
(at most 32 additions in a lane, 8 over lanes, in the root mean square below 7 of them) as for the RMS norm; they move y by that over the deviation.  With mu = mean |r| / deviation,
y is off by at most 16 * 2^-24 (|y - bias| + (1 + mu) |weight|) + 2^-24 |y|; a result in bfloat16 is rounded to 8 significant bits, 2^-8 of it at most.
Gradients: the same relative to the terms that are added up, whose sizes the reference gives.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 16 * 2.0 ** -24
EPS = 1e-5
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def make(rows, cols, dtype, seed=0, shift=0.7):
    g = torch.Generator().manual_seed(seed)
    t = lambda: ((torch.randn(rows, cols, generator=g) + shift * torch.randn(rows, 1, generator=g)) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)
    return dict(x=t(), residual=t(), weight=1 + 0.3 * torch.randn(cols, generator=g), bias=0.5 * torch.randn(cols, generator=g), dy=t(), dr=t())


def definition(p, with_residual, with_weight, with_bias, dtype):
    cols = p["x"].shape[1]
    r = (p["x"].float() + p["residual"].float()).to(dtype).double() if with_residual else p["x"].double()
    r = r.requires_grad_(True)
    w = (p["weight"] if with_weight else torch.ones(cols)).double().requires_grad_(True)
    b = (p["bias"] if with_bias else torch.zeros(cols)).double().requires_grad_(True)
    m = r.mean(1, keepdim=True)
    s = torch.sqrt((r - m).pow(2).mean(1, keepdim=True) + EPS)
    return r, w, b, s, (r - m) / s * w + b


SIZES = [(1, 1), (3, 7), (5, 16), (33, 64), (9, 100), (130, 128), (17, 200), (7, 256), (4, 500), (66, 512), (5, 1000), (3, 1023), (6, 2048), (2, 3001), (3, 4096), (2, 8191), (2, 8192),
         (5000, 64), (3000, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("with_residual,with_weight,with_bias", [(True, True, True), (False, True, True), (True, False, True), (False, True, False), (True, False, False)])
@pytest.mark.parametrize("node", ["c++", "python"])
def test_forward_and_backward(rows, cols, dtype, with_residual, with_weight, with_bias, node, monkeypatch):
    from paper_2507_08637_amd import autograd
    if node == "python":
        monkeypatch.setattr(autograd, "_node", False)
    p = make(rows, cols, dtype, rows + cols)
    g = {k: t.cuda() for k, t in p.items()}
    x = g["x"].requires_grad_(True)
    weight = g["weight"].requires_grad_(True) if with_weight else None
    bias = g["bias"].requires_grad_(True) if with_bias else None
    residual = g["residual"].requires_grad_(True) if with_residual else None
    leaves = [t for t in (x, weight, bias, residual) if t is not None]
    r64, w64, b64, s64, y64 = definition(p, with_residual, with_weight, with_bias, dtype)
    if with_residual:
        y, r = autograd.wersa_layer_norm(x, weight, bias, residual, eps=EPS)
        assert torch.equal(r.detach().double().cpu(), r64.detach())
        grads = torch.autograd.grad((y, r), leaves, (g["dy"], g["dr"]))
        want_r, want_w, want_b = torch.autograd.grad((y64, r64 * 1), (r64, w64, b64), (p["dy"].double(), p["dr"].double()))
        assert torch.equal(grads[0], grads[-1])
    else:
        y = autograd.wersa_layer_norm(x, weight, bias, eps=EPS)
        grads = torch.autograd.grad(y, leaves, g["dy"])
        want_r, want_w, want_b = torch.autograd.grad(y64, (r64, w64, b64), p["dy"].double())
    r64, w64, b64, s64, y64 = (t.detach() for t in (r64, w64, b64, s64, y64))
    mu = r64.abs().mean(1, keepdim=True) / s64          # what the mean's roundings are worth in deviations
    bound = F32 * ((y64 - b64).abs() + (1 + mu) * w64.abs()) + 1.01 * ROUND[dtype] * y64.abs() + 1e-30
    assert ((y.detach().double().cpu() - y64).abs() <= bound).all()
    dy = p["dy"].double()
    hat = (r64 - r64.mean(1, keepdim=True)) / s64
    # dx is a difference of three terms: roundings act on each, of a size that the difference may be far below
    gy = (dy * w64).abs().amax(1, keepdim=True) / s64
    size = gy * (1 + mu) * (2 + hat.abs()) * math.sqrt(cols)
    err = (grads[0].double().cpu() - want_r).abs()
    assert (err <= 1.01 * ROUND[dtype] * want_r.abs() + 4 * F32 * (size + want_r.abs()) + 1e-30).all()
    if with_weight:
        terms = (dy.abs() * (hat.abs() + F32 / 16 * (1 + mu))).norm(dim=0) + (dy.abs() * (1 + mu)).sum(0) / 16
        assert ((grads[1].double().cpu() - want_w).abs() <= 64 * 2.0 ** -24 * (terms + want_w.abs()) + 1e-30).all()
    if with_bias:
        got = grads[2 if with_weight else 1]
        assert ((got.double().cpu() - want_b).abs() <= 64 * 2.0 ** -24 * (dy.norm(dim=0) + want_b.abs()) + 1e-30).all()


def test_gradients_against_differences():
    """float32 with steps of 1e-2: the differences of a smooth function in float64 are right to 1e-4 of its scale."""
    from paper_2507_08637_amd import autograd
    p = make(6, 40, torch.float32, 3)
    g = {k: t.cuda() for k, t in p.items()}
    leaves = [g[k].requires_grad_(True) for k in ("x", "weight", "bias", "residual")]
    y, r = autograd.wersa_layer_norm(g["x"], g["weight"], g["bias"], g["residual"], eps=EPS)
    grads = torch.autograd.grad((y, r), leaves, (g["dy"], g["dr"]))

    def loss(q):
        _, _, _, _, y64 = definition(dict(p, x=q["x"].double() + q["residual"].double(), weight=q["weight"], bias=q["bias"]), False, True, True, torch.float64)
        return float((y64.detach() * p["dy"].double()).sum() + ((q["x"].double() + q["residual"].double()) * p["dr"].double()).sum())
    gen = torch.Generator().manual_seed(9)
    for name, grad in zip(("x", "weight", "bias", "residual"), grads):
        way = torch.randn(p[name].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        q = {k: v.double() for k, v in p.items()}
        up, down = dict(q, **{name: q[name] + h * way}), dict(q, **{name: q[name] - h * way})
        slope, got = (loss(up) - loss(down)) / (2 * h), float((grad.double().cpu() * way).sum())
        assert abs(slope - got) <= 1e-4 * float((grad.double().cpu() * way).abs().sum()), name


def test_rows_far_from_zero():
    """mean(r^2) - mean(r)^2 would have nothing left of these."""
    from paper_2507_08637_amd import binding
    g = torch.Generator().manual_seed(1)
    x = 4096 + torch.randn(50, 512, generator=g)
    y, _, stats = binding.wersa_layer_norm_forward(x.cuda(), eps=0.0, want_stats=True)
    m = x.double().mean(1, keepdim=True)
    s = (x.double() - m).pow(2).mean(1, keepdim=True).sqrt()
    want = (x.double() - m) / s
    # the mean's roundings: F32 of 4096 at most, over a deviation of about 1; centred values are exact to half a unit of 4096's last place
    assert ((y.double().cpu() - want).abs() <= F32 * (want.abs() + 4100 / s)).all()
    assert ((stats[:, 0].double().cpu() - m[:, 0]).abs() <= F32 * 4100).all()
    assert ((stats[:, 1].double().cpu() * s[:, 0] - 1).abs() <= F32 * (2 + 4100 / 512)).all()


def test_constant_rows():
    """A deviation of zero: eps alone keeps the row finite, and y is the bias."""
    from paper_2507_08637_amd import autograd
    x = torch.full((4, 96), 2.5, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    b = torch.randn(96, device="cuda")
    y = autograd.wersa_layer_norm(x, None, b)
    assert torch.equal(y, b.bfloat16().expand(4, 96))
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
    assert (dx == 0).all()


def test_strided_rows_streams_and_not_a_number():
    from paper_2507_08637_amd import binding
    p = {k: t.cuda() for k, t in make(40, 96, torch.bfloat16).items()}
    wide = torch.zeros(40, 301, dtype=torch.bfloat16, device="cuda")
    x, res = wide[:, 1:97], wide[:, 150:246]
    x.copy_(p["x"])
    res.copy_(p["residual"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, r, _ = binding.wersa_layer_norm_forward(x, p["weight"], p["bias"], residual=res, stream=side)
    side.synchronize()
    want, want_r, _ = binding.wersa_layer_norm_forward(p["x"], p["weight"], p["bias"], residual=p["residual"])
    assert torch.equal(y, want) and torch.equal(r, want_r)
    p["x"][3, 5], p["x"][7, 2] = float("nan"), float("inf")
    z, _, _ = binding.wersa_layer_norm_forward(p["x"], p["weight"], p["bias"])
    fine = [i for i in range(40) if i not in (3, 7)]
    assert torch.isfinite(z[fine]).all() and z[3].isnan().all() and z[7].isnan().all()


def test_no_rows():
    from paper_2507_08637_amd import autograd
    x, w, b = torch.empty(0, 64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
    y = autograd.wersa_layer_norm(x, w, b)
    dx, dw, db = torch.autograd.grad(y.sum(), (x, w, b))
    assert y.shape == (0, 64) and dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("node", ["c++", "python"])
def test_leading_dimensions_and_unused_outputs(node, monkeypatch):
    from paper_2507_08637_amd import autograd
    if node == "python":
        monkeypatch.setattr(autograd, "_node", False)
    p = {k: t.cuda() for k, t in make(24, 64, torch.float32).items()}
    x, b, res = p["x"].view(2, 3, 4, 64).requires_grad_(True), p["bias"].requires_grad_(True), p["residual"].view(2, 3, 4, 64).requires_grad_(True)
    y, r = autograd.wersa_layer_norm(x, p["weight"], b, res)
    assert y.shape == x.shape and r.shape == x.shape
    (dx,) = torch.autograd.grad(r, x, p["dr"].view_as(r), retain_graph=True)
    assert torch.equal(dx.view(24, 64), p["dr"])
    (db,) = torch.autograd.grad(y, b, torch.ones((), device="cuda").expand_as(y), retain_graph=True)     # (the weight wants none)
    assert torch.equal(db, torch.full_like(db, 24))
    (dres,) = torch.autograd.grad(y, res, torch.ones_like(y), retain_graph=True)
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
    assert torch.equal(dx, dres)
    with pytest.raises(RuntimeError):
        y, r = autograd.wersa_layer_norm(x, p["weight"], b, res)
        (d,) = torch.autograd.grad(y.square().sum(), x, create_graph=True)
        torch.autograd.grad(d.sum(), x)
