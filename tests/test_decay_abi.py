"""Host-side checks of the causal operators' entry points and binding, without a GPU: bad arguments come back as error codes before anything is launched."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    from paper_2507_08637_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_08637_amd import build
        build.build()
    return binding.load_library()


def desc(**kw):
    from paper_2507_08637_amd.binding import WersaDecayDesc
    f = dict(dict(B=2, H=3, n=100, dk=64, dv=32, dtype=1, packed=0, scale=0.125), **kw)
    H, n = max(1, f["H"]), max(1, f["n"])
    three = ctypes.c_int64 * 3
    for name, d in (("q", f["dk"]), ("k", f["dk"]), ("v", f["dv"]), ("o", f["dv"])):
        f.setdefault("stride_" + name, three(H * n * d, n * d, d))
    return WersaDecayDesc(**f)


ONE = ctypes.c_void_p(1 << 20)   # never dereferenced
HUGE = 1 << 40


def forward(lib, d, q=ONE, k=ONE, v=ONE, ld=ONE, offsets=None, init=None, fin=None, slots=None, rows=2, out=ONE, saved=None, ws=ONE, wb=HUGE):
    return lib.wersa_decay_forward(None if d is None else ctypes.byref(d), q, k, v, ld, offsets, init, fin, slots, rows, out, saved, ws, wb, None)


three = ctypes.c_int64 * 3


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 1), (dict(H=0), 1), (dict(n=-1), 1), (dict(dk=0), 1), (dict(dv=-16), 1), (dict(dtype=5), 1), (dict(packed=2), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(stride_q=three(6400, -1, 64)), 1), (dict(stride_k=three(19200, 0, 64)), 1),
    (dict(stride_v=three(0, 3200, 32)), 1), (dict(stride_o=three(9600, 3200, 16)), 1),
    (dict(dk=24), 2), (dict(dv=8), 2), (dict(dk=144), 2), (dict(dv=256), 2), (dict(H=70000), 2), (dict(B=70000), 2), (dict(n=(1 << 30) + 1), 2),
])
def test_bad_descriptors(lib, kw, status):
    d = desc(**kw)
    assert forward(lib, d) == status
    assert lib.wersa_decay_saved_bytes(ctypes.byref(d)) == 0 and lib.wersa_decay_workspace_bytes(ctypes.byref(d), 1) == 0
    assert lib.wersa_decay_backward(ctypes.byref(d), *[ONE] * 4, None, None, ONE, None, *[ONE] * 4, None, ONE, HUGE, None) == status


def test_bad_arguments(lib):
    d = desc()
    assert forward(lib, None) == 1
    for name in ("q", "k", "v", "ld", "out"):
        assert forward(lib, d, **{name: None}) == 1, name
    assert forward(lib, d, offsets=ONE) == 1 and forward(lib, desc(packed=1)) == 1     # offsets exactly where sequences are packed
    assert forward(lib, d, init=ctypes.c_void_p(8)) == 1 and forward(lib, d, fin=ctypes.c_void_p(1028)) == 1
    assert forward(lib, d, init=ONE, rows=1) == 1 and forward(lib, d, fin=ONE, slots=ONE, rows=0) == 1
    assert forward(lib, d, saved=ctypes.c_void_p(264)) == 3
    long = desc(B=1, H=1, n=100000)
    need = lib.wersa_decay_saved_bytes(ctypes.byref(long))
    assert need > 64 * 32 * 4
    assert forward(lib, long, ws=None, wb=0) == 3 and forward(lib, long, wb=1024) == 3 and forward(lib, long, ws=ctypes.c_void_p(264)) == 3
    back = lambda d, saved=ONE, ws=ONE, wb=HUGE, dq=ONE, dout=ONE: lib.wersa_decay_backward(
        ctypes.byref(d), ONE, ONE, ONE, ONE, None, None, dout, None, saved, dq, ONE, ONE, None, ws, wb, None)
    assert back(long, saved=None) == 1 and back(long, dq=None) == 1 and back(long, dout=None) == 1
    assert back(long, ws=None) == 3 and back(long, wb=1024) == 3 and back(long, saved=ctypes.c_void_p(264)) == 3
    step = lambda d, state=ONE, slots=None, rows=2, q=ONE: lib.wersa_decay_step(ctypes.byref(d), q, ONE, ONE, ONE, state, slots, rows, ONE, None)
    one = desc(n=1)
    assert step(d) == 1                                                # more than one row
    assert step(one, state=None) == 1 and step(one, q=None) == 1 and step(one, rows=1) == 1
    assert step(one, state=ctypes.c_void_p(8)) == 1 and step(one, slots=ONE, rows=0) == 1
    assert step(desc(n=1, packed=1)) == 1 and step(desc(n=1, dk=24)) == 2


def norm(**kw):
    from paper_2507_08637_amd.binding import WersaNormDesc
    return WersaNormDesc(**dict(dict(rows=10, cols=64, dtype=1, eps=1e-6, stride_x=64, stride_residual=64), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 1), (dict(cols=0), 1), (dict(dtype=2), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(stride_x=63), 1),
    (dict(stride_residual=0), 1), (dict(cols=8193, stride_x=8193, stride_residual=8193), 2), (dict(rows=(1 << 31) + 1), 2),
])
def test_norm_refuses(lib, kw, status):
    d = ctypes.byref(norm(**kw))
    assert lib.wersa_rms_norm_forward(d, ONE, None, None, None, ONE, None, None) == status
    assert lib.wersa_rms_norm_eight_bit(d, ONE, None, None, None, ONE, ONE, None) == status
    assert lib.wersa_rms_norm_backward(d, ONE, None, ONE, ONE, None, ONE, ONE, ONE, HUGE, None) == status
    assert lib.wersa_rms_norm_workspace_bytes(d) == 0


def test_norm_arguments(lib):
    d = ctypes.byref(norm())
    assert lib.wersa_rms_norm_forward(None, ONE, None, None, None, ONE, None, None) == 1
    assert lib.wersa_rms_norm_forward(d, None, None, None, None, ONE, None, None) == 1
    assert lib.wersa_rms_norm_forward(d, ONE, None, None, None, None, None, None) == 1
    assert lib.wersa_rms_norm_forward(d, ONE, ONE, None, None, ONE, None, None) == 1          # a residual, and no buffer for the stream
    assert lib.wersa_rms_norm_eight_bit(d, ONE, None, None, None, ONE, None, None) == 1       # no scales
    need = lib.wersa_rms_norm_workspace_bytes(d)
    back = lambda r=ONE, rstd=ONE, dy=ONE, dx=ONE, dw=ONE, ws=ONE, wb=HUGE: lib.wersa_rms_norm_backward(d, r, None, rstd, dy, None, dx, dw, ws, wb, None)
    assert back(r=None) == 1 and back(rstd=None) == 1 and back(dy=None) == 1 and back(dx=None) == 1
    assert need > 0 and back(wb=need - 4) == 3 and back(ws=None) == 3 and back(ws=ctypes.c_void_p(264)) == 3


def test_binding_refuses():
    """Shapes, types and layouts, before the library is called."""
    from paper_2507_08637_amd import binding
    q, v, ld = torch.zeros(2, 3, 10, 32), torch.zeros(2, 3, 10, 16), torch.zeros(3)
    bad = [
        dict(q=q[0]), dict(q=q.double()), dict(q=q.bfloat16()), dict(v=v[:, :, :9]), dict(v=v[:, :2]), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)),
        dict(log_decay=ld[:2]), dict(log_decay=ld.double()), dict(out=v[:, :, :, :8]), dict(offsets=torch.tensor([0, 5], dtype=torch.int32)),
        dict(initial_state=torch.zeros(2, 3, 16, 32)), dict(initial_state=torch.zeros(1, 3, 32, 16)), dict(initial_state=torch.zeros(2, 3, 32, 16).bfloat16()),
        dict(slots=torch.zeros(2, dtype=torch.int64)), dict(slots=torch.zeros(3, dtype=torch.int32)), dict(slots=torch.zeros(2, dtype=torch.int32), want_state=True),
    ]
    for kw in bad:
        args = dict(dict(q=q, k=q, v=v, log_decay=ld), **kw)
        with pytest.raises((AssertionError, TypeError)):
            binding.wersa_decay_forward(**args)
    half = q.half()
    with pytest.raises(TypeError):
        binding.wersa_decay_forward(half, half, v.half(), ld)
    x = torch.zeros(4, 8)
    for kw in (dict(weight=torch.zeros(7)), dict(weight=torch.zeros(8).double()), dict(residual=x[:3]), dict(residual=x.bfloat16()), dict(y=x.bfloat16())):
        with pytest.raises((AssertionError, TypeError)):
            binding.wersa_rms_norm_forward(x, **kw)
    with pytest.raises(AssertionError):
        binding.wersa_rms_norm_forward(x.t())
    with pytest.raises(TypeError):
        binding.wersa_rms_norm_forward(x.half())


def test_tensors_of_the_host_are_refused():
    """Their addresses would fault on the GPU."""
    from paper_2507_08637_amd import autograd, binding
    q, v, ld = torch.zeros(2, 3, 10, 32), torch.zeros(2, 3, 10, 16), torch.zeros(3)
    for call in (lambda: binding.wersa_decay_forward(q, q, v, ld), lambda: autograd.wersa_decay_attention(q, q, v, ld),
                 lambda: binding.wersa_decay_step(q[:, :, 0], q[:, :, 0], v[:, :, 0], ld, torch.zeros(2, 3, 32, 16)),
                 lambda: binding.wersa_decay_backward(q, q, v, ld, v, torch.zeros(64)),
                 lambda: binding.wersa_rms_norm_forward(q.view(-1, 32)), lambda: binding.wersa_rms_norm_eight_bit(q.view(-1, 32)),
                 lambda: autograd.wersa_rms_norm(q), lambda: binding.wersa_rms_norm_backward(q.view(-1, 32), torch.zeros(60), q.view(-1, 32))):
        with pytest.raises(AssertionError, match="GPU"):
            call()
