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
