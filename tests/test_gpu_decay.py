"""Causal linear attention with a decay for each head against its definition in float64 (every pair of a row and an earlier one).

Tolerances (relative in the 2-norm, per output).  float32 outputs and states: every sum is in float32 with at most 64 products in a chunk and one addition per
chunk and segment, each rounding 2^-24 of the sum so far and of either sign: 64 * 2^-24 = 4e-6 leaves a factor of eight to sqrt(64) of them.
bfloat16 outputs: three roundings to 8 significant bits (the weights of a chunk's rows, the state as an operand, the result), 2^-8 at worst and below
2^-9 in the root mean square, of either sign: sqrt(3) 2^-9 < 2^-8.
Single elements, of their own size or the root mean square of their row or of all: eight standard deviations of that, of which there is one in 10^15.  (The terms of
an element are of the size of its row, whatever they cancel to: rows of a walk that begins with a large state are larger than the rest.)
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOL = {torch.float32: 64 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def close(got, want, dtype, what):
    got, want = got.detach().double().cpu(), want.detach().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    if not want.numel():
        return
    err, tol = got - want, TOL[dtype]
    norm = float(want.norm())
    assert float(err.norm()) <= tol * norm + 1e-30, (what, float(err.norm()) / (norm + 1e-300))
    rms = norm / math.sqrt(want.numel())
    row = want.pow(2).mean(-1, keepdim=True).sqrt().clamp(min=rms)
    assert float((err.abs() - 8 * tol * torch.maximum(want.abs(), row)).max()) <= 1e-30, (what, "element")


def definition(q, k, v, ld, scale, S0=None):
    """(H, n, d) float64 on the CPU: output and final state."""
    n = q.shape[1]
    t = torch.arange(n, dtype=torch.float64)
    rel = (t[:, None] - t[None, :])
    power = lambda e: torch.where(e == 0, torch.ones(()).double(), torch.exp(e.clamp(min=0) * ld.clamp(min=-1e4)[:, None, None]))
    A = torch.where(rel >= 0, power(rel[None]), torch.zeros(()).double()) * (q @ k.transpose(1, 2))
    out = scale * (A @ v)
    final = (k * power((n - 1 - t)[None, :, None])).transpose(1, 2) @ v
    if S0 is not None:
        out = out + scale * power((t + 1)[None, :, None]) * (q @ S0)
        final = final + power(torch.full((1, 1, 1), float(n), dtype=torch.float64)) * S0
    return out, final


def decays(H, kind="geometric"):
    if kind == "geometric":
        return torch.log1p(-torch.exp2(-5 - 3 * torch.arange(H, dtype=torch.float32) / max(1, H - 1)))
    if kind == "strong":      # powers that leave float32 within a chunk, a decay of zero, and none at all
        return torch.tensor(([-5.0, -float("inf"), 0.0, -0.5] * H)[:H])
    raise ValueError(kind)


def make(B, H, n, dk, dv, dtype, seed=0, layout="bhnd", state=False, kind="geometric", grads=False):
    g = torch.Generator().manual_seed(seed)
    def tensor(d):
        x = torch.randn(B, H, n, d, generator=g).to(dtype)
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if layout == "bnhd" else x
    p = dict(q=tensor(dk), k=tensor(dk), v=tensor(dv), ld=decays(H, kind), S0=None)
    if state:
        p["S0"] = torch.randn(B, H, dk, dv, generator=g)
    if grads:
        p["dout"] = tensor(dv)
        p["dfinal"] = torch.randn(B, H, dk, dv, generator=g)
    return p


def to(p, dev="cuda"):
    return {k: x.to(dev) if torch.is_tensor(x) else x for k, x in p.items()}


def reference(p, scale, lengths=None, grads=False):
    """Per sequence; packed ones with their lengths.  Returns out, final and with grads dq, dk, dv, dS0 in float64."""
    wide = {n: p[n].double().requires_grad_(grads and n != "ld") for n in ("q", "k", "v", "S0", "ld") if p[n] is not None}
    S0 = wide.get("S0")
    outs, finals, at = [], [], 0
    for b in range(p["q"].shape[0] if lengths is None else len(lengths)):
        rows = (b,) if lengths is None else (0, slice(None), slice(at, at + lengths[b]))
        at += 0 if lengths is None else lengths[b]
        o, f = definition(*(wide[x][rows] for x in "qkv"), wide["ld"], scale, None if S0 is None else S0[b])
        outs.append(o)
        finals.append(f)
    res = dict(out=torch.stack(outs) if lengths is None else torch.cat(outs, 1)[None], final=torch.stack(finals))
    if grads:
        leaves = [wide[x] for x in ("q", "k", "v", "S0") if x in wide]
        res.update(zip(("dq", "dk", "dv", "dS0"), torch.autograd.grad((res["out"], res["final"]), leaves, (p["dout"].double(), p["dfinal"].double()))))
    return res


SIZES = [  # B, H, n, dk, dv
    (1, 1, 1, 16, 16), (2, 3, 2, 64, 64), (1, 2, 63, 64, 64), (3, 1, 64, 32, 48), (1, 3, 65, 64, 128), (2, 2, 127, 128, 64), (1, 2, 200, 128, 128),
    (1, 1, 1000, 64, 64), (1, 2, 1537, 128, 128), (1, 1, 700, 48, 80), (2, 1, 517, 16, 112), (800, 1, 70, 16, 16),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,n,dk,dv", SIZES)
@pytest.mark.parametrize("state", [False, True])
def test_forward(B, H, n, dk, dv, dtype, state):
    from paper_2507_08637_amd import binding
    p = make(B, H, n, dk, dv, dtype, seed=n, state=state, layout="bnhd" if n % 2 else "bhnd")
    g = to(p)
    out, final, _ = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], initial_state=g["S0"], want_state=True)
    ref = reference(p, dk ** -0.5)
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,n,dk,dv", SIZES)
@pytest.mark.parametrize("state", [False, True])
def test_backward(B, H, n, dk, dv, dtype, state):
    from paper_2507_08637_amd import binding
    p = make(B, H, n, dk, dv, dtype, seed=n + 1, state=state, grads=True, layout="bhnd" if n % 2 else "bnhd")
    g = to(p)
    _, _, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], scale=0.3, initial_state=g["S0"], want_state=True, want_saved=True)
    got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, scale=0.3, initial_state=g["S0"],
                                       dfinal_state=g["dfinal"], want_dinitial=True)
    ref = reference(p, 0.3, grads=True)
    for name in ("dq", "dk", "dv"):
        close(got[name], ref[name], dtype, name)
    if state:
        close(got["dinitial_state"], ref["dS0"], torch.float32, "dS0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,dk,dv", [(40, 16, 32), (300, 64, 64), (600, 128, 128)])
def test_decays_of_any_size(n, dk, dv, dtype):
    from paper_2507_08637_amd import binding
    p = make(1, 4, n, dk, dv, dtype, seed=5, state=True, kind="strong", grads=True)
    g = to(p)
    out, final, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], initial_state=g["S0"], want_state=True, want_saved=True)
    got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, initial_state=g["S0"], dfinal_state=g["dfinal"],
                                       want_dinitial=True)
    ref = reference(p, dk ** -0.5, grads=True)
    for h in range(4):
        close(out[:, h], ref["out"][:, h], dtype, "out")
        close(final[:, h], ref["final"][:, h], torch.float32, "final")
        for name in ("dq", "dk", "dv"):
            close(got[name][:, h], ref[name][:, h], dtype, name)


LENGTHS = [[1], [0, 1], [5, 0, 64, 1, 65, 130, 0], [700, 1, 3, 900, 256], [64] * 9, [0, 0, 300], [1024, 1, 0]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("H,dk,dv", [(1, 64, 64), (3, 128, 128), (40, 16, 48)])
def test_packed(lengths, H, dk, dv, dtype):
    from paper_2507_08637_amd import binding
    if H == 40:
        lengths = [x * 2 for x in lengths]
    n, B = sum(lengths), len(lengths)
    p = make(1, H, n, dk, dv, dtype, seed=n, layout="bnhd", grads=True)
    gen = torch.Generator().manual_seed(1)
    p["S0"], p["dfinal"] = torch.randn(B, H, dk, dv, generator=gen), torch.randn(B, H, dk, dv, generator=gen)
    g = to(p)
    offsets = torch.tensor([sum(lengths[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    common = dict(scale=0.2, offsets=offsets, initial_state=g["S0"])
    out, final, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], want_state=True, want_saved=True, **common)
    got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, dfinal_state=g["dfinal"], want_dinitial=True, **common)
    ref = reference(p, 0.2, lengths, grads=True)
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name in ("dq", "dk", "dv"):
        close(got[name], ref[name], dtype, name)
    close(got["dinitial_state"], ref["dS0"], torch.float32, "dS0")
    # each sequence as it is alone: neighbours do not reach it
    at = 0
    for b, length in enumerate(lengths):
        rows = slice(at, at + length)
        at += length
        alone, _, _ = binding.wersa_decay_forward(*(g[x][:, :, rows] for x in "qkv"), g["ld"], scale=0.2, initial_state=g["S0"][b:b + 1].contiguous())
        close(out[:, :, rows], alone.double().cpu(), dtype, "alone")


def test_offsets_that_leave_rows_out():
    """Rows of no sequence are not written, and offsets past the tensor end with it."""
    from paper_2507_08637_amd import binding
    p = to(make(1, 2, 300, 64, 64, torch.bfloat16))
    out = torch.full_like(p["v"], 7.0)
    offsets = torch.tensor([20, 150, 400], dtype=torch.int32, device="cuda")
    binding.wersa_decay_forward(p["q"], p["k"], p["v"], p["ld"], offsets=offsets, out=out)
    assert (out[:, :, :20] == 7).all()
    for rows in (slice(20, 150), slice(150, 300)):
        want, _, _ = binding.wersa_decay_forward(*(p[x][:, :, rows] for x in "qkv"), p["ld"])
        close(out[:, :, rows], want.double().cpu(), torch.bfloat16, "rows")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 16, 16), (3, 2, 64, 64), (5, 7, 48, 80), (2, 3, 128, 128), (40, 8, 64, 128), (300, 1, 128, 112), (260, 1, 32, 16)])
def test_step(B, H, dk, dv, dtype):
    from paper_2507_08637_amd import binding
    p = make(B, H, 1, dk, dv, dtype, seed=B, state=True)
    g = to(p)
    state = g["S0"].clone()
    out = binding.wersa_decay_step(g["q"][:, :, 0], g["k"][:, :, 0], g["v"][:, :, 0], g["ld"], state)
    ref = reference(p, dk ** -0.5)
    close(out, ref["out"][:, :, 0], dtype, "out")
    close(state, ref["final"], torch.float32, "state")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_slots(dtype):
    """States in a cache: prompts leave theirs in their slots, tokens go on from there, a sequence without a slot has zeros and touches nothing."""
    from paper_2507_08637_amd import binding
    B, H, n, d, rows = 4, 2, 90, 64, 9
    p = make(B, H, n + 1, d, d, dtype, seed=3)
    g = to(p)
    cache = torch.full((rows, H, d, d), 3.0, device="cuda")
    slots = torch.tensor([7, -1, 2, rows], dtype=torch.int32, device="cuda")
    first = [g[x][:, :, :n].contiguous() for x in "qkv"]
    _, final, _ = binding.wersa_decay_forward(*first, g["ld"], final_state=cache, slots=slots)
    assert final is cache
    ref = reference({**p, **{x: p[x][:, :, :n] for x in "qkv"}}, d ** -0.5)
    for b, s in ((0, 7), (2, 2)):
        close(cache[s], ref["final"][b], torch.float32, "state")
    others = [s for s in range(rows) if s not in (7, 2)]
    assert (cache[others] == 3).all()
    out = binding.wersa_decay_step(*(g[x][:, :, n] for x in "qkv"), g["ld"], cache, slots=slots)
    ref = reference(p, d ** -0.5)
    for b, s in ((0, 7), (2, 2)):
        close(out[b], ref["out"][b, :, n], dtype, "out")
        close(cache[s], ref["final"][b], torch.float32, "state")
    assert (out[[1, 3]] == 0).all() and (cache[others] == 3).all()
    # on from the cache, in place
    before = cache.clone()
    out, _, _ = binding.wersa_decay_forward(*first, g["ld"], initial_state=cache, final_state=cache, slots=slots)
    S0 = torch.zeros(B, H, d, d)
    S0[0], S0[2] = before[7].cpu(), before[2].cpu()
    ref = reference({**p, **{x: p[x][:, :, :n] for x in "qkv"}, "S0": S0}, d ** -0.5)
    close(out, ref["out"], dtype, "out")
    for b, s in ((0, 7), (2, 2)):
        close(cache[s], ref["final"][b], torch.float32, "state")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows(dtype):
    from paper_2507_08637_amd import binding
    p = to(make(2, 3, 0, 64, 32, dtype, state=True))
    out, final, saved = binding.wersa_decay_forward(p["q"], p["k"], p["v"], p["ld"], initial_state=p["S0"], want_state=True, want_saved=True)
    assert out.shape == (2, 3, 0, 32) and torch.equal(final, p["S0"])
    g = binding.wersa_decay_backward(p["q"], p["k"], p["v"], p["ld"], out, saved, initial_state=p["S0"], dfinal_state=p["S0"], want_dinitial=True)
    assert torch.equal(g["dinitial_state"], p["S0"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [100, 900])
def test_strides_alignment_and_streams(n, dtype):
    """Slices of a fused projection that begins at an odd element, on a stream of its own."""
    from paper_2507_08637_amd import binding
    B, H, dk, dv = 2, 3, 48, 32
    p = make(B, H, n, dk, dv, dtype, seed=9, grads=True)
    width = H * (2 * dk + dv) + 5
    fused = torch.zeros(B * n * width + 1, dtype=dtype, device="cuda")[1:].view(B, n, width)
    at, views = 1, {}
    for name, d in (("q", dk), ("k", dk), ("v", dv)):
        views[name] = fused[:, :, at:at + H * d].unflatten(2, (H, d)).transpose(1, 2)
        views[name].copy_(p[name])
        at += H * d
    g = to(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty(B, n, H, dv, dtype=dtype, device="cuda").transpose(1, 2)
    with torch.cuda.stream(side):
        _, final, saved = binding.wersa_decay_forward(views["q"], views["k"], views["v"], g["ld"], out=out, want_state=True, want_saved=True)
        got = binding.wersa_decay_backward(views["q"], views["k"], views["v"], g["ld"], g["dout"], saved, dfinal_state=g["dfinal"], want_dinitial=True)
    side.synchronize()
    p["S0"] = torch.zeros(B, H, dk, dv)
    ref = reference(p, dk ** -0.5, grads=True)
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name in ("dq", "dk", "dv"):
        close(got[name], ref[name], dtype, name)
    close(got["dinitial_state"], ref["dS0"], torch.float32, "dS0")


@pytest.mark.parametrize("n", [130, 1100])
def test_the_future_does_not_reach_back(n):
    from paper_2507_08637_amd import binding
    p = to(make(1, 2, n, 64, 64, torch.bfloat16, seed=4))
    run = lambda: binding.wersa_decay_forward(p["q"], p["k"], p["v"], p["ld"])[0].clone()
    before = run()
    cut = n - 40
    for x in "qkv":
        p[x][:, :, cut:] *= -3
    after = run()
    assert torch.equal(before[:, :, :cut], after[:, :, :cut]) and not torch.equal(before[:, :, cut:], after[:, :, cut:])


def test_results_are_the_same_every_time():
    from paper_2507_08637_amd import binding
    p = to(make(1, 2, 3000, 64, 64, torch.bfloat16, seed=4, grads=True))
    def run():
        out, final, saved = binding.wersa_decay_forward(p["q"], p["k"], p["v"], p["ld"], want_state=True, want_saved=True)
        g = binding.wersa_decay_backward(p["q"], p["k"], p["v"], p["ld"], p["dout"], saved, dfinal_state=p["dfinal"], want_dinitial=True)
        return [out, final] + list(g.values())
    a, b = run(), run()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_offsets_of_elements_beyond_32_bits():
    """Rows 2^24 elements apart: the last one lies 2^31 elements behind the first."""
    from paper_2507_08637_amd import binding
    n, step = 130, 1 << 24
    p = make(1, 1, n, 64, 64, torch.bfloat16, seed=8)
    pool = torch.empty((n - 1) * step + 4 * 64, dtype=torch.bfloat16, device="cuda")
    views = {name: pool.as_strided((1, 1, n, 64), (64, 64, step, 1), 64 * i) for i, name in enumerate("qkvo")}
    for x in "qkv":
        views[x].copy_(p[x])
    _, final, _ = binding.wersa_decay_forward(views["q"], views["k"], views["v"], p["ld"].cuda(), out=views["o"], want_state=True)
    ref = reference(p, 0.125)
    close(views["o"], ref["out"], torch.bfloat16, "out")
    close(final, ref["final"], torch.float32, "final")


def test_gradients_against_differences():
    """float32, central differences of a loss in float64 of the definition are in test_backward's reference; here of the operator itself."""
    from paper_2507_08637_amd import autograd
    p = to(make(1, 2, 90, 16, 32, torch.float32, seed=2, state=True, grads=True))
    leaves = {x: p[x].clone().requires_grad_(True) for x in ("q", "k", "v", "S0")}
    def loss(**at):
        x = {**{n: t.detach() for n, t in leaves.items()}, **at}
        out, final = autograd.wersa_decay_attention(x["q"], x["k"], x["v"], p["ld"], initial_state=x["S0"])
        return (out.double() * p["dout"]).sum() + (final.double() * p["dfinal"]).sum()
    grads = torch.autograd.grad(loss(**leaves), list(leaves.values()))
    gen = torch.Generator(device="cuda").manual_seed(0)
    for (name, x), grad in zip(leaves.items(), grads):
        d = torch.randn(x.shape, generator=gen, device="cuda")
        # the loss is linear in each of them: no truncation; its value carries 2^-24 of each of its terms
        step = 1.0
        diff = (loss(**{name: x.detach() + step * d}) - loss(**{name: x.detach() - step * d})) / (2 * step)
        slope = (grad.double() * d).sum()
        size = float(grad.double().norm() * d.norm())
        assert abs(float(diff - slope)) <= 64 * 2.0 ** -24 * size, (name, float(diff), float(slope))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_autograd(dtype):
    """Through the node: broadcast values, an output that is not used, a state that needs no gradient, an expanded incoming gradient."""
    from paper_2507_08637_amd import autograd
    B, H, n, d = 2, 3, 150, 64
    p = make(B, H, n, d, d, dtype, seed=12, grads=True)
    g = to(p)
    q, k = g["q"].requires_grad_(True), g["k"].requires_grad_(True)
    v1 = g["v"][:, :1].clone().requires_grad_(True)
    out, final = autograd.wersa_decay_attention(q, k, v1.expand(B, H, n, d), g["ld"], scale=0.1)
    one = torch.ones((), dtype=dtype, device="cuda")
    dq, dk, dv = torch.autograd.grad(out, (q, k, v1), one.expand_as(out))
    p["v"], p["dout"], p["S0"] = p["v"][:, :1].expand(B, H, n, d), torch.ones(B, H, n, d), torch.zeros(B, H, d, d)
    p["dfinal"] = torch.zeros(B, H, d, d)
    ref = reference(p, 0.1, grads=True)
    close(out, ref["out"], dtype, "out")
    close(dq, ref["dq"], dtype, "dq")
    close(dk, ref["dk"], dtype, "dk")
    close(dv, ref["dv"].sum(1, keepdim=True), dtype, "dv")   # (three roundings in the sum's terms, one after it)
    out, final = autograd.wersa_decay_attention(q, k, v1.expand(B, H, n, d), g["ld"], scale=0.1)
    dq, dk = torch.autograd.grad(final, (q, k), g["dfinal"])
    assert (dq == 0).all() and torch.isfinite(dk).all() and (dk != 0).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,dk,dv", [(60, 32, 32), (130, 64, 64), (150, 128, 128), (130, 48, 112), (700, 64, 64)])
def test_what_is_not_finite_stays_on_its_side_of_the_mask(n, dk, dv, dtype):
    """Keys and values that are not numbers or not finite in later rows, queries and gradients in earlier ones: rows that do not reach them are as without them."""
    from paper_2507_08637_amd import binding
    p = to(make(1, 2, n, dk, dv, dtype, seed=6, grads=True))
    def run():
        out, final, saved = binding.wersa_decay_forward(p["q"], p["k"], p["v"], p["ld"], want_state=True, want_saved=True)
        g = binding.wersa_decay_backward(p["q"], p["k"], p["v"], p["ld"], p["dout"], saved, dfinal_state=p["dfinal"], want_dinitial=True)
        return dict(out=out, **{x: g[x] for x in ("dq", "dk", "dv")})
    cut = n - 37
    clean = {x: p[x].clone() for x in ("q", "k", "v", "dout")}
    for x, bad in (("v", float("nan")), ("v", float("inf")), ("k", float("inf")), ("k", float("nan"))):
        p.update({x: t.clone() for x, t in clean.items()})
        p[x][:, :, cut + 3] = 0
        want = run()
        p[x][:, :, cut + 3] = bad
        got = run()
        rows = slice(0, cut + 3)
        assert torch.equal(got["out"][:, :, rows], want["out"][:, :, rows]), (x, bad)
        assert torch.equal(got["dq"][:, :, rows], want["dq"][:, :, rows]), (x, bad)
        if x == "v":
            assert not torch.isfinite(got["out"][:, :, cut + 3]).any()
    for x, bad in (("dout", float("nan")), ("dout", -float("inf")), ("q", float("nan")), ("q", float("inf"))):
        p.update({x: t.clone() for x, t in clean.items()})
        p[x][:, :, 21] = 0
        want = run()
        p[x][:, :, 21] = bad
        got = run()
        for name in ("dk", "dv"):
            assert torch.equal(got[name][:, :, 22:], want[name][:, :, 22:]), (x, bad, name)
        if x == "dout":
            assert not torch.isfinite(got["dv"][:, :, 21]).any()


@pytest.mark.parametrize("B,H,dk,dv", [(128, 17, 128, 128), (600, 14, 64, 64)])
def test_step_of_many_states(B, H, dk, dv):
    """More states than the last-level cache keeps: the variant that passes it by."""
    from paper_2507_08637_amd import binding
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    q, k, v, state = normal(B, H, dk), normal(B, H, dk), normal(B, H, dv), normal(B, H, dk, dv)
    ld = decays(H).cuda()
    want = ld.exp().double().view(H, 1, 1) * state.double() + k.double().unsqueeze(3) * v.double().unsqueeze(2)
    out = binding.wersa_decay_step(q, k, v, ld, state, scale=0.5)
    close(state, want.cpu(), torch.float32, "state")
    close(out, (0.5 * (q.double().unsqueeze(3) * want).sum(2)).cpu(), torch.float32, "out")


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orders_of_the_grid(dtype, layout):
    """Heads apart in memory or side by side, in several segments."""
    from paper_2507_08637_amd import binding
    p = make(2, 3, 700, 64, 64, dtype, seed=31, layout=layout, state=True, grads=True)
    g, ref = to(p), reference(p, 0.125, grads=True)
    out, final, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], 0.125, initial_state=g["S0"], want_state=True, want_saved=True)
    got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, 0.125, initial_state=g["S0"], dfinal_state=g["dfinal"], want_dinitial=True)
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name in ("dq", "dk", "dv"):
        close(got[name], ref[name], dtype, name)
    close(got["dinitial_state"], ref["dS0"], torch.float32, "dS0")


def test_more_sequences_than_a_grid_has_in_its_second_dimension():
    """65535 packed sequences of no, one or two rows, heads side by side."""
    from paper_2507_08637_amd import binding
    H, d, B = 2, 64, 65535
    g = torch.Generator().manual_seed(32)
    lengths = torch.randint(0, 3, (B,), generator=g)
    ends = torch.cumsum(lengths, 0)
    n = int(ends[-1])
    q, k, v = (torch.randn(1, n, H, d, generator=g).cuda().permute(0, 2, 1, 3) for _ in range(3))
    ld = decays(H).cuda()
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), ends]).int().cuda()
    out = binding.wersa_decay_forward(q, k, v, ld, 0.125, offsets=offsets)[0]
    second = torch.zeros(n, dtype=torch.bool)
    second[ends[lengths == 2] - 1] = True
    wide = [x.double().cpu()[0] for x in (q, k, v)]
    want = (wide[0] * wide[1]).sum(-1, keepdim=True) * wide[2]
    before = [x.roll(1, 1) for x in wide]
    want += torch.where(second[None, :, None], ld.double().cpu().exp()[:, None, None] * (wide[0] * before[1]).sum(-1, keepdim=True) * before[2], 0.)
    close(out[0], 0.125 * want, torch.float32, "out")


def test_tensors_that_pass_the_caches():
    """A batch whose q, k and v together are larger than the last-level cache against its halves, which are not."""
    from paper_2507_08637_amd import autograd
    g = torch.Generator(device="cuda").manual_seed(33)
    x = [torch.randn(2, 70000, 8, 64, generator=g, device="cuda", dtype=torch.bfloat16).permute(0, 2, 1, 3) for _ in range(4)]
    ld = decays(8).cuda()

    def step(*t):
        leaves = [y.detach().requires_grad_() for y in t[:3]]
        out = autograd.wersa_decay_attention(*leaves, ld, 0.125)[0]
        return [out.detach()] + list(torch.autograd.grad(out, leaves, t[3]))

    whole, halves = step(*x), [step(*(y[i:i + 1] for y in x)) for i in range(2)]
    for a, b, what in zip(whole, zip(*halves), ("out", "dq", "dk", "dv")):
        close(a, torch.cat(b).double().cpu(), torch.bfloat16, what)   # (both have the same roundings, up to the order of a state's sums and where the last chunks begin)
