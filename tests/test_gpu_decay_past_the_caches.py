"""Batches whose q, k and v together are larger than the last-level cache, at widths of 128: against their halves, which are not, forward and backward."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_decay import close, decays


@pytest.mark.parametrize("dk,dv,n", [(128, 128, 25000), (64, 128, 38000), (128, 64, 30000)])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_whole_and_halves(dk, dv, n, layout):
    from paper_2507_08637_amd import autograd
    H = 8
    assert 2 * n * H * (2 * dk + dv) * 2 > 256 << 20 > n * H * (2 * dk + dv) * 2
    g = torch.Generator(device="cuda").manual_seed(34)

    def tensor(d):
        x = torch.randn(2, n, H, d, generator=g, device="cuda", dtype=torch.bfloat16).permute(0, 2, 1, 3)
        return x if layout == "bnhd" else x.contiguous()
    x, ld = [tensor(dk), tensor(dk), tensor(dv), tensor(dv)], decays(H).cuda()

    def step(*t):
        leaves = [y.detach().requires_grad_() for y in t[:3]]
        out = autograd.wersa_decay_attention(*leaves, ld)[0]
        return [out.detach()] + list(torch.autograd.grad(out, leaves, t[3]))
    whole, halves = step(*x), [step(*(y[i:i + 1] for y in x)) for i in range(2)]
    for a, b, what in zip(whole, zip(*halves), ("out", "dq", "dk", "dv")):
        close(a, torch.cat(b).double().cpu(), torch.bfloat16, what)   # (both have the same roundings, up to the order of a state's sums and where the last chunks begin)
