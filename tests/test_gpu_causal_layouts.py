"""Decay attention on layouts other than dense ones: what a program's slices, transposes and broadcasts leave.  Reference and tolerances are those of the operators' other tests."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_decay import close, make, reference, to


@pytest.fixture(params=["c++", "python"])
def node(request, monkeypatch):
    from paper_2507_08637_amd import autograd
    if request.param == "python":
        monkeypatch.setattr(autograd, "_node", False)
    else:
        assert autograd._load_node()
    return autograd


def lone_rows(x, stride):
    """(B, H, 1, d) with the same values and a row stride of `stride` elements."""
    B, H, _, d = x.shape
    y = torch.as_strided(torch.empty(B * H * d, dtype=x.dtype, device=x.device), (B, H, 1, d), (H * d, d, stride, 1))
    y.copy_(x)
    assert y.stride(2) == stride
    return y


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("stride", [0, 1, 16, (1 << 24) + 16, 1 << 27, 1 << 32])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (48, 112), (128, 128)])
def test_a_lone_row_may_have_any_stride(stride, dk, dv, dtype):
    """Less than the width, none, or one whose bytes wrap in 32 bits within a chunk's rows: the state has this row once, and the outputs are its own."""
    from paper_2507_08637_amd import binding
    p = make(2, 3, 1, dk, dv, dtype, seed=20, state=True, grads=True)
    ref = reference(p, 0.3, grads=True)
    g = to(p)
    for x in ("q", "k", "v", "dout"):
        g[x] = lone_rows(g[x], stride)
    out, final, saved = binding.wersa_decay_forward(g["q"], g["k"], g["v"], g["ld"], 0.3, initial_state=g["S0"], want_state=True, want_saved=True)
    got = binding.wersa_decay_backward(g["q"], g["k"], g["v"], g["ld"], g["dout"], saved, 0.3, initial_state=g["S0"], dfinal_state=g["dfinal"], want_dinitial=True)
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name in ("dq", "dk", "dv"):
        close(got[name], ref[name], dtype, name)
    close(got["dinitial_state"], ref["dS0"], torch.float32, "dS0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lone_rows_as_programs_have_them(node, dtype):
    """A column turned into a row (stride 1, and contiguous() leaves it), the first of expanded rows (stride 0), one row of one packed sequence."""
    H, d = 3, 64
    p = make(2, H, 1, d, d, dtype, seed=21, grads=True)
    p["S0"] = torch.zeros(2, H, d, d)
    g = to(p)
    column = lambda x: x[:, :, 0].clone()[..., None].mT
    assert column(g["q"]).stride(2) == 1
    expanded = lambda x: x.expand(2, H, 512, d)[:, :, :1]
    assert expanded(g["k"]).stride(2) == 0
    ref = reference(p, 0.125, grads=True)
    for view in (column, expanded):
        leaves = [view(g[x]).detach().requires_grad_(True) for x in "qkv"]
        out, final = node.wersa_decay_attention(*leaves, g["ld"])
        grads = torch.autograd.grad((out, final), leaves, (view(g["dout"]), g["dfinal"]))
        close(out, ref["out"], dtype, "out")
        close(final, ref["final"], torch.float32, "final")
        for name, x in zip(("dq", "dk", "dv"), grads):
            close(x, ref[name], dtype, name)
    one = {x: t[:1] if x in ("q", "k", "v", "dout", "S0", "dfinal") else t for x, t in p.items()}
    ref = reference(one, 0.125, grads=True)
    leaves = [column(g[x][:1]).detach().requires_grad_(True) for x in "qkv"]
    out, final = node.wersa_decay_attention(*leaves, g["ld"], offsets=torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    grads = torch.autograd.grad((out, final), leaves, (g["dout"][:1], g["dfinal"][:1]))
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name, x in zip(("dq", "dk", "dv"), grads):
        close(x, ref[name], dtype, name)


def check_against_copies(node, leaves, ld, dout, dfinal, dtype):
    """The operator on views against the definition of their values; returns out and the gradients."""
    values = {x: t.detach().cpu().contiguous() for x, t in zip("qkv", leaves)}
    p = dict(values, ld=ld.cpu(), S0=torch.zeros(dfinal.shape), dout=dout.detach().cpu(), dfinal=dfinal.cpu())
    ref = reference(p, 0.125, grads=True)
    out, final = node.wersa_decay_attention(*leaves, ld, 0.125)
    grads = torch.autograd.grad((out, final), leaves, (dout, dfinal))
    close(out, ref["out"], dtype, "out")
    close(final, ref["final"], torch.float32, "final")
    for name, x in zip(("dq", "dk", "dv"), grads):
        close(x, ref[name], dtype, name)
    return (out, *grads)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [100, 700])
def test_windows_that_overlap(node, n, dtype):
    """Sliding windows over the rows of one tensor as the batch, and heads that share columns: outputs and gradients have memory of their own for each."""
    H, d, B = 3, 64, 4
    g = torch.Generator(device="cuda").manual_seed(22)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)
    ld = torch.tensor([-0.1, -0.02, -0.005], device="cuda")
    windows = lambda: normal(n + (B - 1) * (n // 2), H, d).unfold(0, n, n // 2).permute(0, 1, 3, 2)
    assert windows().shape == (B, H, n, d) and windows().stride(0) == n // 2 * H * d
    shared = lambda: normal(B, n, d + 32 * (H - 1)).unfold(2, d, 32).transpose(1, 2)
    assert shared().shape == (B, H, n, d) and shared().stride(1) == 32
    for views in ([windows(), windows(), windows()], [shared(), shared(), shared()], [windows(), shared(), normal(B, H, n, d)]):
        leaves = [x.detach().requires_grad_(True) for x in views]
        for made in check_against_copies(node, leaves, ld, normal(B, H, n, d), torch.randn(B, H, d, d, generator=g, device="cuda"), dtype):
            assert made.untyped_storage().nbytes() == made.numel() * made.element_size()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_slices_of_a_fused_projection(node, dtype):
    """Outputs and gradients hold their own elements, not what lies between the slices, in the projection's order: the output is rows of heads without a copy."""
    from paper_2507_08637_amd import binding
    B, n, H, d = 2, 150, 3, 64
    g = torch.Generator(device="cuda").manual_seed(23)
    fused = torch.randn(B, n, 3, H, d, generator=g, device="cuda").to(dtype)
    q, k, v = (x.detach().requires_grad_(True) for x in fused.permute(2, 0, 3, 1, 4).unbind(0))
    ld = torch.tensor([-0.1, -0.02, -0.005], device="cuda")
    dout, dfinal = torch.randn(B, n, H, d, generator=g, device="cuda").to(dtype).transpose(1, 2), torch.randn(B, H, d, d, generator=g, device="cuda")
    made = check_against_copies(node, (q, k, v), ld, dout, dfinal, dtype)
    for x in made:
        assert x.untyped_storage().nbytes() == x.numel() * x.element_size()
        assert x.transpose(1, 2).is_contiguous()
    with torch.no_grad():
        out, _, saved = binding.wersa_decay_forward(q, k, v, ld, 0.125, want_saved=True)
        grads = binding.wersa_decay_backward(q, k, v, ld, dout, saved, 0.125, dfinal_state=dfinal)
        # into gradients of other strides, slices of a gradient of the whole
        whole = torch.full((B, n, 3, H, d), float("nan"), device="cuda", dtype=dtype)
        into = dict(zip(("dq", "dk", "dv"), whole.permute(2, 0, 3, 1, 4).unbind(0)), dinitial_state=None)
        binding.wersa_decay_backward(q, k, v, ld, dout, saved, 0.125, dfinal_state=dfinal, grads=into)
    assert torch.equal(out, made[0]) and out.transpose(1, 2).is_contiguous()
    for name, x, part in zip(("dq", "dk", "dv"), made[1:], whole.unbind(2)):
        assert torch.equal(grads[name], x) and torch.equal(part.transpose(1, 2), x) and grads[name].transpose(1, 2).is_contiguous()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_heads_that_share_keys_and_values(dtype):
    """The binding on keys and values that are expanded over heads, sequences or rows: as on copies of them, gradients for each of the heads."""
    from paper_2507_08637_amd import binding
    B, H, n, d = 2, 4, 200, 64
    p = to(make(B, H, n, d, d, dtype, seed=24, grads=True))
    common = [p["k"][:, :1], p["v"][:1, :1], p["dout"][:, :, :1]]
    k, v, dout = (x.expand(B, H, n, d) for x in common)
    side = torch.cuda.Stream()

    def run(k, v, dout, stream=None):
        side.wait_stream(torch.cuda.current_stream())
        out, final, saved = binding.wersa_decay_forward(p["q"], k, v, p["ld"], want_state=True, want_saved=True, stream=stream)
        got = binding.wersa_decay_backward(p["q"], k, v, p["ld"], dout, saved, dfinal_state=p["dfinal"], want_dinitial=True, stream=stream)
        state = p["dfinal"].clone()
        side.wait_stream(torch.cuda.current_stream())
        token = binding.wersa_decay_step(p["q"][:, :, 3], k[:, :, 3], v[:, :, 3], p["ld"], state, stream=stream)
        torch.cuda.synchronize()
        return [out, final, *got.values(), token, state]
    want = run(k.contiguous(), v.contiguous(), dout.contiguous())
    for stream in (None, side):
        for a, b in zip(run(k, v, dout, stream), want):
            assert torch.equal(a, b)
