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


Q, V, LD = torch.zeros(2, 3, 10, 32), torch.zeros(2, 3, 10, 16), torch.zeros(3)
STATE, SLOTS = torch.zeros(2, 3, 32, 16), torch.zeros(2, dtype=torch.int32)
SHAPES, DTYPE, COLUMNS, DECAY, STATES = "expect q, k", "share a dtype|must be float32 or bfloat16", "contiguous last dim", "log_decay: float32, one per head", "states are contiguous float32"


def refused(calls, call, match, error=AssertionError):
    with pytest.raises(error, match=match):
        call()
    assert not [name for name in calls if not name.endswith("_bytes")]


def decay(**kw):
    from paper_2507_08637_amd import binding
    return binding.wersa_decay_forward(**dict(dict(q=Q, k=Q, v=V, log_decay=LD), **kw))


@pytest.mark.parametrize("kw,match,error", [
    (dict(q=Q[0]), SHAPES, AssertionError), (dict(k=Q[:, :, :9]), SHAPES, AssertionError), (dict(v=V[:, :, :9]), SHAPES, AssertionError),
    (dict(v=V[:, :2]), SHAPES, AssertionError), (dict(out=V[..., :8]), SHAPES, AssertionError),
    (dict(q=Q.bfloat16()), DTYPE, AssertionError), (dict(out=V.bfloat16()), DTYPE, AssertionError), (dict(q=Q.half(), k=Q.half(), v=V.half()), DTYPE, TypeError),
    (dict(q=Q.transpose(2, 3).contiguous().transpose(2, 3)), COLUMNS, AssertionError),
    (dict(log_decay=LD[:2]), DECAY, AssertionError), (dict(log_decay=LD.double()), DECAY, AssertionError), (dict(log_decay=torch.zeros(6)[::2]), DECAY, AssertionError),
    (dict(offsets=torch.tensor([0, 5], dtype=torch.int32)), "packed sequences", AssertionError),
    (dict(q=Q[:1], k=Q[:1], v=V[:1], offsets=torch.tensor([0, 5])), "packed sequences", AssertionError),
    (dict(q=Q[:1], k=Q[:1], v=V[:1], offsets=torch.tensor([0], dtype=torch.int32)), "packed sequences", AssertionError),
    (dict(initial_state=torch.zeros(2, 3, 16, 32)), STATES, AssertionError), (dict(initial_state=torch.zeros(1, 3, 32, 16)), STATES, AssertionError),
    (dict(final_state=STATE.bfloat16()), STATES, AssertionError), (dict(final_state=torch.zeros(2, 3, 16, 32).mT), STATES, AssertionError),
    (dict(final_state=STATE, slots=SLOTS.long()), "slots: int32", AssertionError), (dict(final_state=STATE, slots=SLOTS[:1]), "slots: int32", AssertionError),
    (dict(initial_state=STATE, final_state=torch.zeros(5, 3, 32, 16), slots=SLOTS), STATES, AssertionError),
    (dict(slots=SLOTS, want_state=True), "buffer of the caller's", AssertionError),
    (dict(saved=torch.zeros(255)), "saved buffer holds", AssertionError),
])
def test_decay_forward(calls, kw, match, error):
    refused(calls, lambda: decay(**kw), match, error)


def test_decay_forward_takes_what_is_right(calls):
    decay()
    decay(initial_state=STATE, want_state=True, want_saved=True)
    decay(final_state=torch.zeros(7, 3, 32, 16), slots=SLOTS)
    decay(q=Q.transpose(1, 2).contiguous().transpose(1, 2), out=torch.zeros(2, 10, 3, 16).transpose(1, 2))
    decay(q=Q[:1], k=Q[:1], v=V[:1], offsets=torch.tensor([0, 5, 5, 10], dtype=torch.int32), initial_state=torch.zeros(3, 3, 32, 16))
    assert calls.count("wersa_decay_forward") == 5


def test_decay_backward(calls):
    from paper_2507_08637_amd import binding
    saved = torch.zeros(256)

    def back(**kw):
        return binding.wersa_decay_backward(**dict(dict(q=Q, k=Q, v=V, log_decay=LD, dout=V, saved=saved), **kw))
    fine = dict(dq=torch.zeros(2, 10, 3, 32).transpose(1, 2), dk=torch.zeros_like(Q), dv=torch.zeros_like(V), dinitial_state=None)
    for name, bad in (("dq", Q[:, :2]), ("dk", Q.bfloat16()), ("dv", torch.zeros(2, 3, 16, 10).mT)):
        refused(calls, lambda: back(grads=dict(fine, **{name: bad})), name + " has its tensor's shape")
    refused(calls, lambda: back(grads=dict(fine, dinitial_state=STATE[:1])), STATES)
    refused(calls, lambda: back(dout=V[..., :8]), SHAPES)
    refused(calls, lambda: back(dout=V.bfloat16()), DTYPE)
    refused(calls, lambda: back(dfinal_state=STATE.double()), STATES)
    refused(calls, lambda: back(saved=saved[:255]), "saved buffer holds")
    refused(calls, lambda: back(log_decay=LD[:1]), DECAY)
    back(grads=fine)
    back(want_dinitial=True, dfinal_state=STATE)
    assert calls.count("wersa_decay_backward") == 2


def test_decay_step(calls):
    from paper_2507_08637_amd import binding

    def step(**kw):
        return binding.wersa_decay_step(**dict(dict(q=Q[:, :, 0], k=Q[:, :, 0], v=V[:, :, 0], log_decay=LD, state=STATE), **kw))
    refused(calls, lambda: step(q=Q), "expect q, k")
    refused(calls, lambda: step(k=Q[:, :2, 0]), "expect q, k")
    refused(calls, lambda: step(v=V[:, :, 0].bfloat16()), DTYPE)
    refused(calls, lambda: step(q=torch.zeros(2, 32, 3).mT), COLUMNS)
    refused(calls, lambda: step(log_decay=LD[:1]), DECAY)
    refused(calls, lambda: step(state=STATE[:1]), STATES)
    refused(calls, lambda: step(state=STATE, slots=SLOTS.long()), "slots: int32")
    step()
    step(state=torch.zeros(9, 3, 32, 16), slots=SLOTS)
    assert calls.count("wersa_decay_step") == 2


@pytest.mark.parametrize("name", ["wersa_rms_norm_forward", "wersa_rms_norm_eight_bit"])
def test_norm(calls, name):
    from paper_2507_08637_amd import binding
    entry, x = getattr(binding, name), torch.zeros(4, 8)
    for kw, match in ((dict(weight=torch.zeros(7)), "weight: float32"), (dict(weight=torch.zeros(8).double()), "weight: float32"), (dict(residual=x[:3]), "x's shape and dtype"),
                      (dict(residual=x.bfloat16()), "x's shape and dtype"), (dict(y=torch.zeros(4, 8, dtype=torch.float16)), "y is dense"), (dict(residual=x, r=torch.zeros(8, 4).t()), "r is dense")):
        refused(calls, lambda: entry(x, **kw), match)
    refused(calls, lambda: entry(x.view(2, 2, 8)), "contiguous columns")
    refused(calls, lambda: entry(torch.zeros(8, 4).t()), "contiguous columns")
    refused(calls, lambda: entry(x.half()), "must be float32 or bfloat16", TypeError)
    entry(x)
    entry(torch.zeros(4, 20)[:, 3:11], torch.ones(8), residual=x)
    assert calls == [name] * 2
