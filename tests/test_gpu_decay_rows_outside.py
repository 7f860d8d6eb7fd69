"""Packed sequences that leave rows out, as padded batches have them: such rows are zeros in what the operator allocates, and what they hold reaches nothing.
The other rows are compared with the definition at the tolerances of the operators' other tests."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_decay import close, make, reference, to

NAN = float("nan")


@pytest.fixture(params=["c++", "python", "binding"])
def step(request, monkeypatch):
    """Forward and backward: out, final states, gradients of q, k, v and the initial states."""
    from paper_2507_08637_amd import autograd, binding
    if request.param == "binding":
        def run(g, offsets):
            common = dict(scale=0.2, offsets=offsets, initial_state=g["S0"])
            out, final, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], want_state=True, want_saved=True, **common)
            spoilt = {name: torch.full_like(g[x], NAN) for name, x in (("dq", "q"), ("dk", "k"), ("dv", "v"))}    # of an earlier call
            spoilt["dinitial_state"] = torch.full_like(g["S0"], NAN)
            got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, dfinal_state=g["dfinal"], grads=spoilt, **common)
            return [out, final] + [got[x] for x in ("dq", "dk", "dv", "dinitial_state")]
        return run
    if request.param == "python":
        monkeypatch.setattr(autograd, "_node", False)
    else:
        assert autograd._load_node()

    def run(g, offsets):
        leaves = [g[x].detach().requires_grad_(True) for x in ("q", "k", "v", "S0")]
        out, final = autograd.wersa_decay_attention(*leaves[:3], g["ld"], 0.2, leaves[3], offsets)
        return [out.detach(), final.detach(), *torch.autograd.grad((out, final), leaves, (g["dout"], g["dfinal"]))]
    return run


def spoil_free_memory(like):
    """What the allocator hands out next holds NaN."""
    blocks = [torch.full_like(x, NAN, memory_format=torch.contiguous_format) for x in like for _ in range(3)]
    torch.cuda.synchronize()
    del blocks


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("H,dk,dv", [(2, 64, 64), (3, 128, 128), (2, 48, 16)])
@pytest.mark.parametrize("n,cuts", [(300, [20, 150, 260]), (300, [0, 7, 299]), (300, [299, 299, 300]), (1500, [700, 700, 1400]), (1500, [1, 2, 1500]), (64, [0, 0, 0]), (64, [64, 64, 64])])
def test_rows_outside_are_zeros(step, n, cuts, H, dk, dv, layout, dtype):
    p = make(1, H, n, dk, dv, dtype, seed=n + cuts[0], layout=layout, grads=True)
    gen = torch.Generator().manual_seed(2)
    p["S0"], p["dfinal"] = torch.randn(2, H, dk, dv, generator=gen), torch.randn(2, H, dk, dv, generator=gen)
    inside = slice(cuts[0], cuts[-1])
    outside = [slice(0, cuts[0]), slice(cuts[-1], n)]
    ref = reference({x: t[:, :, inside] if x in ("q", "k", "v", "dout") else t for x, t in p.items()}, 0.2, [b - a for a, b in zip(cuts, cuts[1:])], grads=True)
    for x in ("q", "k", "v", "dout"):
        for rows in outside:
            p[x][:, :, rows] = NAN
    g = to(p)
    spoil_free_memory([g[x] for x in ("q", "k", "v", "dout")])
    got = step(g, torch.tensor(cuts, dtype=torch.int32, device="cuda"))
    for x, name in zip(got, ("out", "final", "dq", "dk", "dv", "dS0")):
        if name in ("final", "dS0"):
            close(x, ref[name], torch.float32, name)
            continue
        for rows in outside:
            assert (x[:, :, rows] == 0).all(), name
        close(x[:, :, inside], ref[name], dtype, name)


def test_a_projection_under_a_masked_loss():
    """The gradient of the weights that q, k and v come from: padded rows, whatever is in their memory, add nothing to it."""
    from paper_2507_08637_amd import autograd
    g = torch.Generator(device="cuda").manual_seed(0)
    n, H, d, hidden = 400, 2, 32, 64
    x, w = torch.randn(n, hidden, generator=g, device="cuda"), torch.randn(hidden, 3 * H * d, generator=g, device="cuda") / 8
    ld = torch.tensor([-0.1, -0.01], device="cuda")

    def gradient(x, offsets):
        spoil_free_memory([x.new_empty(1, H, len(x), d)] * 4)
        weight = w.clone().requires_grad_(True)
        q, k, v = (x @ weight).view(1, len(x), 3, H, d).permute(2, 0, 3, 1, 4).unbind(0)
        out, _ = autograd.wersa_decay_attention(q, k, v, ld, offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
        out[:, :, offsets[0]:offsets[-1]].square().sum().backward()
        return weight.grad
    close(gradient(x, [50, 200, 330]), gradient(x[50:330].contiguous(), [0, 150, 280]).double().cpu(), torch.float32, "weight")
