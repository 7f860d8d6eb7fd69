"""The norm's autograd entry on layouts other than rows one behind the other: as on dense copies, bit for bit."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(params=["c++", "python"])
def node(request, monkeypatch):
    from paper_2507_08637_amd import autograd
    if request.param == "python":
        monkeypatch.setattr(autograd, "_node", False)
    else:
        assert autograd._load_node()
    return autograd


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["transposed", "one sequence transposed", "a token for all rows", "a token for all sequences", "windows", "one column", "slices"])
def test_any_layout(node, kind, dtype):
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)

    def view():
        if kind == "transposed":
            return normal(96, 40).t()
        if kind == "one sequence transposed":
            return normal(1, 96, 40).transpose(1, 2)
        if kind == "a token for all rows":
            return normal(1, 96).expand(40, 96)
        if kind == "a token for all sequences":
            return normal(1, 5, 96).expand(8, 5, 96)
        if kind == "windows":
            return normal(39 * 32 + 96).unfold(0, 96, 32)
        if kind == "one column":
            return torch.as_strided(normal(40), (40, 1), (1, 7))
        return normal(40, 3, 96)[:, 1]
    x, residual = view(), view()
    weight, dy, dr = torch.randn(x.shape[-1], generator=g, device="cuda"), normal(*x.shape), normal(*x.shape)

    def run(x, residual):
        leaves = [x.detach().requires_grad_(True), weight.clone().requires_grad_(True), residual.detach().requires_grad_(True)]
        y, r = node.wersa_rms_norm(leaves[0], leaves[1], leaves[2])
        alone = node.wersa_rms_norm(leaves[0], leaves[1])
        return [y, r, alone, *torch.autograd.grad((y, r), leaves, (dy, dr)), *torch.autograd.grad(alone, leaves[:2], dy)]
    dense = lambda t: t.clone(memory_format=torch.contiguous_format)
    for a, b in zip(run(x, residual), run(dense(x), dense(residual))):
        assert a.shape == b.shape and torch.equal(a, b)
