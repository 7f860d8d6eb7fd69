"""What the causal operators' Python entry points refuse, each by the check that is meant for it, without a GPU: the check for tensors of the host, which comes last, is left out, and the library
behind it replaced by one that notes its calls."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def calls(monkeypatch):
    """Names of the entry points that are reached."""
    from paper_2507_08637_amd import autograd, binding
    reached = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                reached.append(name)
                return 1024 if name.endswith("_bytes") else 0
            return entry
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "_on_one_gpu", lambda *tensors: None)
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    monkeypatch.setattr(autograd, "_node", False)
    return reached


def test_a_decay_that_wants_a_gradient(calls):
    """It would get none."""
    from paper_2507_08637_amd import autograd
    q, ld = torch.zeros(2, 3, 10, 32), torch.zeros(3, requires_grad=True)
    with pytest.raises(AssertionError, match="log_decay.* has no gradient"):
        autograd.wersa_decay_attention(q, q, q, ld)
    assert not calls
    with torch.no_grad():
        autograd.wersa_decay_attention(q, q, q, ld)
    autograd.wersa_decay_attention(q, q, q, ld.detach())
    assert calls.count("wersa_decay_forward") == 2


def test_a_residual_of_another_shape(calls):
    """As many elements in other dimensions would be added row by row in the wrong order."""
    from paper_2507_08637_amd import autograd
    x = torch.zeros(4, 6, 32)
    for shape in ((6, 4, 32), (24, 32), (2, 12, 32)):
        with pytest.raises(AssertionError, match="x's shape"):
            autograd.wersa_rms_norm(x, residual=torch.zeros(shape))
    assert not calls
    y, r = autograd.wersa_rms_norm(x, residual=torch.zeros(4, 6, 32))
    assert y.shape == r.shape == x.shape and "wersa_rms_norm_forward" in calls
