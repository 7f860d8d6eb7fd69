"""The causal operators' nodes of the autograd graph: the one in C++ and the one in Python make the same calls."""
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


def leaves(*shapes, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(1)
    return [torch.randn(s, generator=g, device="cuda").to(dtype).requires_grad_(True) for s in shapes]


def decay_call(autograd, dtype, packed=False, initial=True):
    q, k, v = leaves((1 if packed else 2, 3, 130, 32), (1 if packed else 2, 3, 130, 32), (1 if packed else 2, 3, 130, 64), dtype=dtype)
    S0 = leaves((2, 3, 32, 64))[0]
    offsets = torch.tensor([0, 47, 130], dtype=torch.int32, device="cuda") if packed else None
    ld = torch.tensor([-0.1, -0.01, -1.0], device="cuda")
    ins = [q, k, v] + ([S0] if initial else [])
    return ins, autograd.wersa_decay_attention(q, k, v, ld, 0.2, S0 if initial else None, offsets)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("packed,initial", [(False, True), (False, False), (True, True)])
def test_decay_nodes_agree_with_the_binding(node, dtype, packed, initial):
    from paper_2507_08637_amd import binding
    ins, (out, final) = decay_call(node, dtype, packed, initial)
    g = torch.Generator(device="cuda").manual_seed(2)
    dout, dfinal = torch.randn(out.shape, generator=g, device="cuda").to(dtype), torch.randn(final.shape, generator=g, device="cuda")
    got = torch.autograd.grad((out, final), ins, (dout, dfinal))
    q, k, v = (x.detach() for x in ins[:3])
    S0 = ins[3].detach() if initial else None
    common = dict(scale=0.2, initial_state=S0, offsets=torch.tensor([0, 47, 130], dtype=torch.int32, device="cuda") if packed else None)
    ld = torch.tensor([-0.1, -0.01, -1.0], device="cuda")
    want_out, want_final, saved = binding.wersa_decay_forward(q, k, v, ld, want_state=True, want_saved=True, **common)
    want = binding.wersa_decay_backward(q, k, v, ld, dout, saved, dfinal_state=dfinal, want_dinitial=initial, **common)
    assert torch.equal(out, want_out) and torch.equal(final, want_final)
    for x, name in zip(got, ("dq", "dk", "dv", "dinitial_state")):
        assert torch.equal(x, want[name]), name


def test_parts_of_the_outputs_and_of_the_inputs(node):
    ins, (out, final) = decay_call(node, torch.float32)
    whole = torch.autograd.grad((out, final), ins, (torch.ones_like(out), torch.zeros_like(final)), retain_graph=True)
    alone = torch.autograd.grad(out, ins, torch.ones((), device="cuda").expand_as(out), retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(whole, alone))
    (dk,) = torch.autograd.grad(final, ins[1], torch.ones_like(final))
    assert torch.isfinite(dk).all() and (dk != 0).any()
    x, w, r = leaves((20, 48), (48,), (20, 48))
    y, stream = node.wersa_rms_norm(x, w, r)
    dx, dr = torch.autograd.grad((y, stream), (x, r), (torch.ones_like(y), torch.ones_like(y)), retain_graph=True)
    assert torch.equal(dx, dr)
    (dw,) = torch.autograd.grad(y, w, torch.ones_like(y))
    y2 = node.wersa_rms_norm(stream.detach(), w)
    assert torch.equal(torch.autograd.grad(y2, w, torch.ones_like(y))[0], dw)
    frozen = node.wersa_rms_norm(x, w.detach(), residual=r.detach())[0]
    one_less = torch.autograd.grad(frozen, x, torch.ones_like(y))[0]     # nothing reaches the stream from elsewhere
    assert torch.allclose(one_less + 1, dx, rtol=2.0 ** -22, atol=2.0 ** -22)
    plain = node.wersa_rms_norm(x.view(4, 5, 48))
    assert plain.shape == (4, 5, 48) and torch.autograd.grad(plain.sum(), x)[0].shape == x.shape


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_saved_tensors_in_another_layout(node, dtype):
    """Hooks that give back copies, dense: the call is described by what is there."""
    q, k, v = (x.transpose(1, 2) for x in leaves((2, 70, 3, 32), (2, 70, 3, 32), (2, 70, 3, 32), dtype=dtype))
    ld = torch.tensor([-0.1, -0.01, -1.0], device="cuda")
    def run():
        out, _ = node.wersa_decay_attention(q, k, v, ld)
        y = node.wersa_rms_norm(out, torch.ones(32, device="cuda"))
        return torch.autograd.grad(y, (q, k, v), torch.ones_like(y))
    want = run()
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x.detach().clone(memory_format=torch.contiguous_format), lambda x: x):
        got = run()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.autograd.graph.save_on_cpu():
        got = run()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_twice_is_refused(node):
    ins, (out, _) = decay_call(node, torch.float32)
    with pytest.raises(RuntimeError):
        g = torch.autograd.grad(out.sum(), ins[0], create_graph=True)[0]
        torch.autograd.grad(g.sum(), ins[1])
    x, w = leaves((5, 32), (32,))
    with pytest.raises(RuntimeError):
        g = torch.autograd.grad(node.wersa_rms_norm(x, w).sum(), x, create_graph=True)[0]
        torch.autograd.grad(g.sum(), x)


def test_refusals(node):
    from paper_2507_08637_amd import binding
    q, k, v = leaves((1, 2, 10, 24), (1, 2, 10, 24), (1, 2, 10, 24))
    with pytest.raises(binding.WersaError):
        node.wersa_decay_attention(q, k, v, torch.zeros(2, device="cuda"))
    with pytest.raises(AssertionError):
        node.wersa_decay_attention(q, k[:, :, :5], v, torch.zeros(2, device="cuda"))
    with pytest.raises(binding.WersaError):
        node.wersa_rms_norm(torch.zeros(2, 9000, device="cuda"))
    with pytest.raises(AssertionError):
        node.wersa_rms_norm(torch.zeros(2, 64, device="cuda"), torch.ones(63, device="cuda"))
    with pytest.raises(TypeError):
        node.wersa_rms_norm(torch.zeros(2, 64, device="cuda", dtype=torch.float16))


def test_one_tensor_of_the_host_among_others_is_refused():
    from paper_2507_08637_amd import binding
    q, k, v = (x.detach() for x in leaves((1, 2, 10, 32), (1, 2, 10, 32), (1, 2, 10, 32)))
    ld, offsets, slots = torch.zeros(2), torch.tensor([0, 4, 10], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    state = torch.zeros(1, 2, 32, 32, device="cuda")
    for call in (lambda: binding.wersa_decay_forward(q, k, v, ld), lambda: binding.wersa_decay_forward(q, k, v, ld.cuda(), offsets=offsets),
                 lambda: binding.wersa_decay_forward(q, k, v, ld.cuda(), final_state=state, slots=slots),
                 lambda: binding.wersa_decay_forward(q, k, v, ld.cuda(), initial_state=state.cpu()),
                 lambda: binding.wersa_decay_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], ld.cuda(), state, slots=slots),
                 lambda: binding.wersa_rms_norm_forward(q[0, 0], torch.ones(32)), lambda: binding.wersa_rms_norm_forward(q[0, 0], residual=q[0, 0].cpu())):
        with pytest.raises(AssertionError, match="GPU"):
            call()
