"""What the recurrence, the embedding, the layer norm and the logits' operator refuse, without a GPU: the Python entry points, each by the check that is meant for it (the library behind
them replaced by one that notes its calls), and the C entry points by their status."""
import ctypes

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
    monkeypatch.setattr(binding, "_on_current_gpu", lambda *tensors: None)
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    monkeypatch.setattr(autograd, "_node", False)
    return reached


def refused(calls, call, match, error=AssertionError):
    with pytest.raises(error, match=match):
        call()
    assert not [name for name in calls if not name.endswith("_bytes")]


X, STATE, SLOTS = torch.zeros(2, 10, 16), torch.zeros(2, 16), torch.zeros(2, dtype=torch.int32)
INT = dict(dtype=torch.int32)
SHAPES, DTYPE, STATES = r"expect x, gate and out \(B, n, C\)", "must share a dtype", "states are contiguous float32"


@pytest.mark.parametrize("kw,match,error", [
    (dict(x=X[0]), SHAPES, AssertionError), (dict(gate=X[:, :9]), SHAPES, AssertionError), (dict(gate=X[..., :8]), SHAPES, AssertionError), (dict(out=X[:1]), SHAPES, AssertionError),
    (dict(gate=X.bfloat16()), DTYPE, AssertionError), (dict(out=X.bfloat16()), DTYPE, AssertionError), (dict(x=X.half(), gate=X.half()), "must be float32 or bfloat16", TypeError),
    (dict(x=torch.zeros(2, 16, 10).mT), "contiguous channels", AssertionError),
    (dict(offsets=torch.tensor([0, 10], **INT)), "packed sequences", AssertionError), (dict(x=X[:1], gate=X[:1], offsets=torch.tensor([0, 10])), "packed sequences", AssertionError),
    (dict(x=X[:1], gate=X[:1], offsets=torch.tensor([0], **INT)), "packed sequences", AssertionError),
    (dict(initial_state=STATE[:1]), STATES, AssertionError), (dict(initial_state=STATE.bfloat16()), STATES, AssertionError), (dict(final_state=torch.zeros(16, 2).t()), STATES, AssertionError),
    (dict(final_state=STATE, slots=SLOTS.long()), "slots: int32", AssertionError), (dict(final_state=STATE, slots=SLOTS[:1]), "slots: int32", AssertionError),
    (dict(initial_state=STATE, final_state=torch.zeros(5, 16), slots=SLOTS), STATES, AssertionError),
    (dict(slots=SLOTS, want_state=True), "buffer of the caller's", AssertionError), (dict(saved=torch.zeros(255)), "saved buffer holds", AssertionError),
])
def test_recurrence_forward(calls, kw, match, error):
    from paper_2507_08637_amd import binding
    refused(calls, lambda: binding.wersa_recurrence_forward(**dict(dict(x=X, gate=X), **kw)), match, error)


def test_recurrence_takes_what_is_right(calls):
    from paper_2507_08637_amd import autograd, binding
    binding.wersa_recurrence_forward(X, X.transpose(0, 1).contiguous().transpose(0, 1), want_state=True, want_saved=True, initial_state=STATE)
    binding.wersa_recurrence_forward(X, X, final_state=torch.zeros(7, 16), slots=SLOTS)
    binding.wersa_recurrence_forward(X[:1], X[:1].expand(1, 10, 16), torch.tensor([0, 5, 5, 10], **INT), initial_state=torch.zeros(3, 16))
    binding.wersa_recurrence_forward(torch.zeros(2, 10, 1).expand(2, 10, 1), torch.zeros(10, 2, 1).transpose(0, 1))
    autograd.wersa_recurrence(X, torch.zeros(2, 16, 10).mT)
    assert calls.count("wersa_recurrence_forward") == 5
    saved = torch.zeros(256)
    binding.wersa_recurrence_backward(X, X, X, saved, want_dinitial=True, dfinal_state=STATE)
    fine = dict(dx=torch.zeros_like(X), dgate=torch.zeros_like(X), dinitial_state=None)
    del calls[:]
    for name, bad, match in (("dx", X[:1], SHAPES), ("dgate", X.bfloat16(), DTYPE), ("dx", torch.zeros(2, 16, 10).mT, "contiguous channels"), ("dinitial_state", STATE[:1], STATES)):
        refused(calls, lambda: binding.wersa_recurrence_backward(X, X, X, saved, grads=dict(fine, **{name: bad})), match)
    refused(calls, lambda: binding.wersa_recurrence_backward(X, X, X[:, :9], saved), SHAPES)
    refused(calls, lambda: binding.wersa_recurrence_backward(X, X, X, saved[:255]), "saved buffer holds")
    refused(calls, lambda: binding.wersa_recurrence_backward(X, X, X, saved, dfinal_state=STATE.double()), STATES)


def test_recurrence_step(calls):
    from paper_2507_08637_amd import binding
    x = X[:, 0]
    refused(calls, lambda: binding.wersa_recurrence_step(X, X, STATE), "expect x, gate and out")
    refused(calls, lambda: binding.wersa_recurrence_step(x, x[:, :8], STATE), "expect x, gate and out")
    refused(calls, lambda: binding.wersa_recurrence_step(x, x.bfloat16(), STATE), DTYPE)
    refused(calls, lambda: binding.wersa_recurrence_step(torch.zeros(16, 2).t(), x, STATE), "contiguous channels")
    refused(calls, lambda: binding.wersa_recurrence_step(x, x, STATE[:1]), STATES)
    refused(calls, lambda: binding.wersa_recurrence_step(x, x, STATE, slots=SLOTS.long()), "slots: int32")
    binding.wersa_recurrence_step(x, x, STATE)
    binding.wersa_recurrence_step(x, x, torch.zeros(9, 16), slots=SLOTS)
    assert calls.count("wersa_recurrence_step") == 2


def test_embedding(calls):
    from paper_2507_08637_amd import autograd, binding
    t, w = torch.zeros(3, 4, dtype=torch.long), torch.zeros(10, 8)
    forward, back = binding.wersa_embedding_forward, binding.wersa_embedding_backward
    refused(calls, lambda: forward(t.float(), w), "tokens: int32 or int64")
    refused(calls, lambda: forward(t.to(torch.int16), w), "tokens: int32 or int64")
    refused(calls, lambda: forward(t, w[0]), r"weight is \(vocabulary, cols\)")
    refused(calls, lambda: autograd.wersa_embedding(t, w[0]), r"weight is \(vocabulary, cols\)")
    refused(calls, lambda: forward(t, torch.zeros(8, 10).t()), "contiguous columns")
    refused(calls, lambda: forward(t, w[:1].expand(10, 8)), "do not share memory")
    refused(calls, lambda: forward(t, w.half()), "must be float32 or bfloat16", TypeError)
    refused(calls, lambda: forward(t, w, dtype=torch.float16), "must be float32 or bfloat16", TypeError)
    refused(calls, lambda: forward(t, w, out=torch.zeros(3, 4, 9)), "out is")
    refused(calls, lambda: forward(t, w, dtype=torch.bfloat16, out=torch.zeros(3, 4, 8)), "another dtype")
    refused(calls, lambda: back(t, torch.zeros(3, 5, 8), 10), "dout is")
    refused(calls, lambda: back(t, torch.zeros(3, 4, 8), 10, dweight=torch.zeros(9, 8)), "dweight is")
    refused(calls, lambda: back(t, torch.zeros(3, 4, 1).expand(3, 4, 8), 10), "contiguous columns")
    forward(t.t(), w, 2.0, torch.bfloat16)
    forward(t.int(), torch.zeros(10, 20)[:, 3:11], out=torch.zeros(3, 4, 11)[..., 2:10])
    back(t, torch.zeros(3, 4, 11)[..., 2:10], 10, dtype=torch.bfloat16)
    assert [n for n in calls if not n.endswith("_bytes")] == ["wersa_embedding_forward"] * 2 + ["wersa_embedding_backward"]


def test_layer_norm(calls):
    from paper_2507_08637_amd import autograd, binding
    x, entry = torch.zeros(4, 8), binding.wersa_layer_norm_forward
    for kw, match in ((dict(weight=torch.zeros(7)), "weight: float32"), (dict(weight=torch.zeros(1, 8)), "weight: float32"), (dict(bias=torch.zeros(7)), "bias: float32"),
                      (dict(bias=torch.zeros(8).double()), "bias: float32"), (dict(bias=torch.zeros(16)[::2]), "bias: float32"), (dict(residual=x[:3]), "x's shape and dtype"),
                      (dict(residual=x.bfloat16()), "x's shape and dtype"), (dict(y=torch.zeros(8, 4).t()), "y is dense"), (dict(stats=torch.zeros(4)), "stats is dense"),
                      (dict(residual=x, r=torch.zeros(4, 9)[:, :8]), "r is dense")):
        refused(calls, lambda: entry(x, **kw), match)
    refused(calls, lambda: entry(torch.zeros(8, 4).t()), "contiguous columns")
    refused(calls, lambda: entry(x.half()), "must be float32 or bfloat16", TypeError)
    with pytest.raises(AssertionError, match="x's shape"):
        autograd.wersa_layer_norm(torch.zeros(4, 6, 8), residual=torch.zeros(6, 4, 8))
    back = binding.wersa_layer_norm_backward
    refused(calls, lambda: back(x, torch.zeros(4), x), "stats is dense")
    refused(calls, lambda: back(x, torch.zeros(4, 2), x.bfloat16()), "dy and dr are dense")
    refused(calls, lambda: back(x, torch.zeros(4, 2), x, dr=torch.zeros(8, 4).t()), "dy and dr are dense")
    refused(calls, lambda: back(x, torch.zeros(4, 2), x, dbias=torch.zeros(9)), "dbias is dense")
    entry(torch.zeros(4, 20)[:, 3:11], torch.ones(8), torch.ones(8), residual=x, want_stats=True)
    back(x, torch.zeros(4, 2), x)
    assert [n for n in calls if not n.endswith("_bytes")] == ["wersa_layer_norm_forward", "wersa_layer_norm_backward"]


def test_logits(calls):
    from paper_2507_08637_amd import binding
    z, h, n = torch.zeros(3, 70), torch.zeros(3, 9, **INT), torch.zeros(3, **INT)
    one, f = torch.ones(3), lambda **kw: binding.wersa_logits_adjust(z, **kw)
    for kw, match in ((dict(out=torch.zeros(3, 71)), "out has"), (dict(out=z.bfloat16()), "out has"), (dict(out=z[:1].expand(3, 70)), "out has"),
                      (dict(history=h), "lengths: int32"), (dict(history=h, lengths=n[:2]), "lengths: int32"), (dict(history=h, lengths=n.long()), "lengths: int32"),
                      (dict(history=h.long(), lengths=n), "history: int32"), (dict(history=h[:2], lengths=n[:2]), "a row for each row"), (dict(history=h.t().contiguous().t(), lengths=n), "history: int32"),
                      (dict(history=h, lengths=n, prompt_lengths=n[:1]), "prompt_lengths: int32"), (dict(history=h, lengths=n, slots=n[:2]), "slots: int32"),
                      (dict(history=h, lengths=n, repetition=one[:2]), "repetition: float32"), (dict(history=h, lengths=n, presence=one.double()), "presence: float32"),
                      (dict(repetition=one), "go by a history"), (dict(lengths=n), "go by a history"), (dict(bias_tokens=h), "biases: int32"),
                      (dict(bias_tokens=h, bias_values=torch.zeros(3, 8)), "biases: int32"), (dict(bias_tokens=h[:2], bias_values=torch.zeros(2, 9)), "biases: int32"),
                      (dict(bias_tokens=h.long(), bias_values=torch.zeros(3, 9)), "biases: int32"), (dict(mask=torch.zeros(3, 2, **INT)), "mask: int32"),
                      (dict(mask=torch.zeros(2, 3, **INT)), "mask: int32"), (dict(mask=torch.zeros(3, 70, dtype=torch.bool)), "mask: int32")):
        refused(calls, lambda: f(**kw), match)
    refused(calls, lambda: binding.wersa_logits_adjust(z[0]), "contiguous columns")
    refused(calls, lambda: binding.wersa_logits_adjust(torch.zeros(70, 3).t()), "contiguous columns")
    refused(calls, lambda: binding.wersa_logits_adjust(z.half()), "must be float32 or bfloat16", TypeError)
    f(history=torch.zeros(8, 9, **INT), lengths=torch.zeros(8, **INT), slots=n, repetition=one, bias_tokens=h[0], bias_values=torch.zeros(9), mask=torch.zeros(3, **INT), out=z)
    binding.wersa_logits_adjust(z[:1].expand(3, 70), mask=torch.zeros(3, 3, **INT))
    assert calls == ["wersa_logits_adjust"] * 2


def test_another_gpu_than_the_current_one(monkeypatch):
    from paper_2507_08637_amd import binding

    class Tensor:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    binding._on_current_gpu(Tensor(0), Tensor(0), None)
    for bad in ((Tensor(1), Tensor(1)), (Tensor(0), Tensor(1)), (Tensor(-1),), (Tensor(0), Tensor(-1))):
        with pytest.raises(AssertionError, match="GPU"):
            binding._on_current_gpu(*bad)


def test_a_stream_is_the_current_one_within_the_call(monkeypatch):
    from paper_2507_08637_amd import binding
    entered = []

    class Guard:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)

        def __exit__(self, *args):
            entered.append("out")
    monkeypatch.setattr(torch.cuda, "stream", Guard)
    call = binding._on_stream(lambda a, b=0: (a, b, list(entered)))
    assert call(1, b=2) == (1, 2, []) and call(3, stream="side") == (3, 0, ["side"]) and entered == ["side", "out"]


# ---- the C entry points: a status before anything is launched ---------------------------------------------

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
ONE = ctypes.c_void_p(1 << 20)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2507_08637_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_08637_amd import build
        build.build()
    return binding.load_library()


def recurrence_desc(**kw):
    from paper_2507_08637_amd.binding import WersaRecurrenceDesc
    d = dict(B=2, n=1000, C=64, dtype=1, packed=0, clear=0, stride_x=(64000, 64), stride_gate=(64000, 64), stride_o=(64000, 64), stride_dx=(64000, 64), stride_dgate=(64000, 64))
    d.update(kw)
    return ctypes.byref(WersaRecurrenceDesc(*[(ctypes.c_int64 * 2)(*v) if isinstance(v, tuple) else v for v in d.values()]))


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(n=-1), INVALID), (dict(C=0), INVALID), (dict(dtype=2), INVALID), (dict(packed=2), INVALID), (dict(clear=-1), INVALID), (dict(stride_x=(-1, 64)), INVALID),
    (dict(stride_gate=(0, -64)), INVALID), (dict(stride_o=(64000, 63)), INVALID), (dict(stride_o=(63999, 64)), INVALID), (dict(stride_o=(64, 64)), INVALID), (dict(packed=1), INVALID),
    (dict(B=65536), UNSUPPORTED), (dict(n=(1 << 30) + 1), UNSUPPORTED), (dict(C=(1 << 20) + 1), UNSUPPORTED), (dict(n=1 << 30, B=60000), UNSUPPORTED)])
def test_recurrence_status(lib, kw, status):
    assert lib.wersa_recurrence_forward(recurrence_desc(**kw), ONE, ONE, None, None, None, None, 0, ONE, None, ONE, 1 << 40, None) == status


def test_recurrence_pointers_and_workspaces(lib):
    d = recurrence_desc()
    size = lib.wersa_recurrence_workspace_bytes(d)
    assert size > 0 and lib.wersa_recurrence_saved_bytes(d) >= 2 * 8 * 64 * 4
    forward = lambda x=ONE, gate=ONE, out=ONE, saved=None, ws=ONE, bytes=size, d=d, **kw: lib.wersa_recurrence_forward(
        d, x, gate, kw.get("offsets"), kw.get("initial"), kw.get("final"), kw.get("slots"), kw.get("rows", 0), out, saved, ws, bytes, None)
    for kw in (dict(x=None), dict(gate=None), dict(out=None), dict(slots=ONE, rows=-1), dict(offsets=ONE)):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(bytes=size - 1), dict(ws=ctypes.c_void_p((1 << 20) + 128)), dict(saved=ctypes.c_void_p((1 << 20) + 4))):
        assert forward(**kw) == WORKSPACE, kw
    # packed initial states that lie where the final ones go are gathered into the workspace, however few rows there are
    short = recurrence_desc(n=10, packed=1)
    assert forward(d=short, offsets=ONE, initial=ONE, final=ONE, ws=None) == WORKSPACE
    back = lambda x=ONE, gate=ONE, dout=ONE, saved=ONE, dx=ONE, dgate=ONE, ws=ONE, bytes=size, d=d: lib.wersa_recurrence_backward(
        d, x, gate, None, None, dout, None, saved, dx, dgate, None, ws, bytes, None)
    for kw in (dict(x=None), dict(gate=None), dict(dout=None), dict(saved=None), dict(dx=None), dict(dgate=None), dict(d=recurrence_desc(stride_dx=(64, 64))),
               dict(d=recurrence_desc(stride_dgate=(0, 0))), dict(d=recurrence_desc(stride_o=(-1, 0)))):
        assert back(**kw) == INVALID, kw
    for kw in (dict(ws=None), dict(bytes=size - 1)):
        assert back(**kw) == WORKSPACE, kw
    step = lambda d, x=ONE, state=ONE, out=ONE: lib.wersa_recurrence_step(d, x, ONE, state, None, 0, out, None)
    for bad in (d, recurrence_desc(n=1, packed=1), recurrence_desc(n=1, stride_o=(63, 0))):
        assert step(bad) == INVALID
    for kw in (dict(x=None), dict(state=None), dict(out=None)):
        assert step(recurrence_desc(n=1), **kw) == INVALID


def embedding_desc(**kw):
    from paper_2507_08637_amd.binding import WersaEmbeddingDesc
    d = dict(tokens=1000, vocabulary=500, cols=64, dtype=1, weight_dtype=0, token_bytes=8, scale=1.0, stride_weight=64, stride_out=64)
    d.update(kw)
    return ctypes.byref(WersaEmbeddingDesc(*d.values()))


def test_embedding_status(lib):
    for kw, status in ((dict(tokens=-1), INVALID), (dict(vocabulary=0), INVALID), (dict(cols=0), INVALID), (dict(dtype=2), INVALID), (dict(weight_dtype=-1), INVALID), (dict(token_bytes=2), INVALID),
                       (dict(stride_weight=63), INVALID), (dict(stride_out=0), INVALID), (dict(tokens=1 << 31), UNSUPPORTED), (dict(cols=(1 << 20) + 1, stride_weight=1 << 21, stride_out=1 << 21), UNSUPPORTED)):
        assert lib.wersa_embedding_forward(embedding_desc(**kw), ONE, ONE, ONE, None) == status, kw
        assert lib.wersa_embedding_backward(embedding_desc(**kw), ONE, ONE, ONE, ONE, 1 << 40, None) == status, kw
        assert lib.wersa_embedding_workspace_bytes(embedding_desc(**kw)) == 0
    d = embedding_desc()
    size = lib.wersa_embedding_workspace_bytes(d)
    for i in range(3):
        args = [None if j == i else ONE for j in range(3)]
        assert lib.wersa_embedding_forward(d, *args, None) == INVALID and lib.wersa_embedding_backward(d, *args, ONE, size, None) == INVALID
    for ws, bytes in ((None, size), (ONE, size - 1), (ctypes.c_void_p((1 << 20) + 128), size)):
        assert lib.wersa_embedding_backward(d, ONE, ONE, ONE, ws, bytes, None) == WORKSPACE


def test_layer_norm_status(lib):
    from paper_2507_08637_amd.binding import WersaNormDesc
    desc = lambda rows=10, cols=64, dtype=0, eps=1e-5, sx=64, sr=64: ctypes.byref(WersaNormDesc(rows, cols, dtype, eps, sx, sr))
    forward = lambda d, x=ONE, res=None, r=None, y=ONE: lib.wersa_layer_norm_forward(d, x, res, None, None, r, y, None, None)
    for kw, status in ((dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(dtype=3), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(sx=63), INVALID), (dict(sr=1), INVALID),
                       (dict(cols=8193, sx=8193, sr=8193), UNSUPPORTED), (dict(rows=(1 << 31) + 1), UNSUPPORTED)):
        assert forward(desc(**kw)) == status, kw
    assert forward(desc(), x=None) == forward(desc(), y=None) == forward(desc(), res=ONE) == INVALID
    size = lib.wersa_layer_norm_workspace_bytes(desc())
    back = lambda r=ONE, stats=ONE, dy=ONE, dx=ONE, dw=ONE, db=ONE, ws=ONE, bytes=size: lib.wersa_layer_norm_backward(desc(), r, None, stats, dy, None, dx, dw, db, ws, bytes, None)
    for name in ("r", "stats", "dy", "dx"):
        assert back(**{name: None}) == INVALID
    for kw in (dict(ws=None), dict(ws=None, dw=None), dict(ws=None, db=None), dict(bytes=size - 1), dict(ws=ctypes.c_void_p((1 << 20) + 16))):
        assert back(**kw) == WORKSPACE, kw


def test_logits_status(lib):
    from paper_2507_08637_amd.binding import WersaLogitsDesc

    def call(logits=ONE, history=None, lengths=None, tokens=None, values=None, out=ONE, **kw):
        d = dict(B=3, vocabulary=100, dtype=0, history_rows=0, history_most=0, biases=0, stride_logits=100, stride_out=100, stride_history=0, stride_bias=0, stride_mask=0)
        d.update(kw)
        return lib.wersa_logits_adjust(ctypes.byref(WersaLogitsDesc(*d.values())), logits, history, lengths, None, None, None, None, None, tokens, values, None, out, None)
    for kw in (dict(B=-1), dict(vocabulary=0), dict(dtype=2), dict(history_rows=-1), dict(history_most=-1), dict(biases=-1), dict(stride_out=99), dict(stride_logits=-1), dict(stride_bias=-1), dict(stride_mask=-1),
               dict(logits=None), dict(out=None), dict(history=ONE), dict(biases=2, tokens=ONE), dict(biases=2, values=ONE), dict(history_rows=3, stride_history=-1)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(B=65536), dict(biases=1024), dict(history_most=1 << 21)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(B=0) == 0
