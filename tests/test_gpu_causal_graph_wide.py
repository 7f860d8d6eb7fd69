"""Decay attention recorded into a HIP graph at the widths whose kernels ask for more LDS than a launch has by default, and with packed sequences that leave rows out."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,offsets", [(900, None), (900, [30, 400, 870]), (90, [0, 40, 80])])
def test_replays(n, offsets, dtype):
    from paper_2507_08637_amd import binding
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)
    q, k, v, dout = (normal(1, 2, n, 128) for _ in range(4))
    ld = torch.tensor([-0.02, -0.3], device="cuda")
    offsets = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")

    def work():
        out, final, saved = binding.wersa_decay_forward(q, k, v, ld, offsets=offsets, want_state=True, want_saved=True)
        grads = binding.wersa_decay_backward(q, k, v, ld, dout, saved, offsets=offsets, want_dinitial=True)
        return [out, final, *grads.values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = work()
    for i in range(3):
        for t in (q, k, v, dout):     # other inputs in the same places, and results that are not there yet
            t.copy_(normal(*t.shape))
        for t in recorded:
            t.fill_(float("nan"))
        want = [t.clone() for t in work()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(recorded, want)), i
