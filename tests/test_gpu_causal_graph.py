"""The causal operators recorded into a HIP graph: replays with other work between them give what eager calls give."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_replays():
    from paper_2507_08637_amd import binding
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    q, k, v, dout = (normal(1, 2, 1000, 64).bfloat16() for _ in range(4))
    q1, k1, v1 = (normal(3, 2, 64).bfloat16() for _ in range(3))
    ld, slots, cache = torch.tensor([-0.02, -0.3], device="cuda"), torch.tensor([4, 1, 2], dtype=torch.int32, device="cuda"), normal(5, 2, 64, 64)
    x, res, w, dy = normal(50, 200).bfloat16(), normal(50, 200).bfloat16(), normal(200), normal(50, 200).bfloat16()

    def work():
        out, final, saved = binding.wersa_decay_forward(q, k, v, ld, want_state=True, want_saved=True)
        grads = binding.wersa_decay_backward(q, k, v, ld, dout, saved, want_dinitial=True)
        token = binding.wersa_decay_step(q1, k1, v1, ld, cache, slots=slots)
        y, r, rstd = binding.wersa_rms_norm_forward(x, w, residual=res, want_rstd=True)
        dx, dw = binding.wersa_rms_norm_backward(r, rstd, dy, w)
        y8, _, scales = binding.wersa_rms_norm_eight_bit(x, w, residual=res)
        return [out, final, *grads.values(), token, y, r, dx, dw, y8.view(torch.uint8), scales]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = work()
    for i in range(4):
        for t in (q, k, v, x, q1, v1):     # other inputs in the same places
            t.copy_(normal(*t.shape))
        start = cache.clone()
        want = [t.clone() for t in work()]
        state = cache.clone()
        cache.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(recorded, want)), i
        assert torch.equal(cache, state)
