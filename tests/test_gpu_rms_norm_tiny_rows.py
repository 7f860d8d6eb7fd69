"""The norm's output in 8 bits where a row is so small that 448 over its largest value leaves float32.

Tolerances: those of the other sizes (half of a step of e4m3, 16 roundings of 2^-24), and for each of y, its largest value and the scale half of the smallest step of float32, 2^-150, which is absolute
down there."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_rms_norm import EPS, F32, e4m3_step


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [7, 64, 513, 3000])
@pytest.mark.parametrize("size", [1e-28, 3e-32, 1e-35, 2e-36, 1e-36, 1e-37, 1e-38, 1e-40])
def test_rows_below_float32s_reciprocals(size, cols, dtype):
    """By small weights, and by small values; zeros among them stay zeros."""
    from paper_2507_08637_amd import binding
    g = torch.Generator().manual_seed(cols)
    x = torch.randn(6, cols, generator=g)
    x[:, ::3] = 0
    x[3] = 0
    by_weight = (x.to(dtype), (1 + 0.3 * torch.randn(cols, generator=g)) * size)
    by_value = ((x * size / EPS ** -0.5).to(dtype), 1 + 0.3 * torch.randn(cols, generator=g))
    for x, weight in (by_weight, by_value):
        r = x.double()
        y64 = r / torch.sqrt(r.pow(2).mean(1, keepdim=True) + EPS) * weight.double()
        most = y64.abs().amax(1)
        y, _, scales = binding.wersa_rms_norm_eight_bit(x.cuda(), weight.cuda(), eps=EPS)
        got = y.double().cpu()
        assert torch.isfinite(got).all() and (got[:, ::3] == 0).all() and (got[3] == 0).all()
        one = torch.ones((), dtype=torch.float64)
        lost = torch.where(most > 0, 448 / most, one)[:, None] * 2 * 2.0 ** -150
        exact = y64 * torch.where(most > 0, 448 / most, one)[:, None]
        assert ((got - exact).abs() <= e4m3_step(exact * (1 + 1e-6) + lost) / 2 + F32 * exact.abs() + lost).all()
        want = torch.where(most > 0, most / 448, one)
        assert ((scales.double().cpu() - want).abs() <= F32 * want + 2.0 ** -150 * (1 + 1 / 448)).all()
