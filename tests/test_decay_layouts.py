"""Layouts that the causal operators' entry points refuse to write, and memory orders that the binding chooses, without a GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests.test_decay_abi import HUGE, ONE, desc, forward, lib, three  # noqa: F401 (lib: the fixture)

# B, H, n = 2, 3, 100, width 32: heads on each other, a sequence that begins within the one before it, rows of heads that meet
OVERLAPPING = [(9600, 16, 96), (3200, 1600, 32), (96, 32, 100), (9600, 3199, 32), (9599, 3200, 32), (3200, 32, 64)]


@pytest.mark.parametrize("strides", OVERLAPPING)
def test_written_tensors_must_not_overlap(lib, strides):  # noqa: F811
    assert forward(lib, desc(stride_o=three(*strides))) == 1
    assert forward(lib, desc(clear=2)) == 1
    back = lambda d: lib.wersa_decay_backward(ctypes.byref(d), *[ONE] * 4, None, None, ONE, None, *[ONE] * 4, None, ONE, HUGE, None)
    for name in ("stride_dq", "stride_dk", "stride_dv"):
        assert back(desc(dk=32, **{name: three(*strides)})) == 1, name
    for tensor in ("stride_q", "stride_k", "stride_v"):     # gradients that are laid out like such a tensor
        assert back(desc(dk=32, **{tensor: three(*strides)})) == 1, tensor
    assert back(desc(dk=32, stride_dq=three(-1, 3200, 32))) == 1 and back(desc(dk=32, stride_dk=three(9600, 3200, (1 << 24) + 32))) == 2   # (rows too far apart)
    step = desc(n=1, stride_o=three(48, 16, 32))
    assert lib.wersa_decay_step(ctypes.byref(step), ONE, ONE, ONE, ONE, ONE, None, 2, ONE, None) == 1


def test_dense_like():
    """What is dense keeps its strides; slices, windows and expanded tensors keep the order of their dimensions."""
    from paper_2507_08637_amd.binding import _dense_like
    x = torch.zeros(2, 3, 10, 16)
    for view in (x, torch.zeros(2, 10, 3, 16).transpose(1, 2), torch.zeros(1, 3, 10, 16), torch.zeros(2, 3, 1, 16)):
        assert _dense_like(view).stride() == view.stride()
    fused = torch.zeros(2, 10, 9, 16)[:, :, 3:6].transpose(1, 2)
    assert _dense_like(fused).stride() == (480, 16, 48, 1)
    windows = torch.zeros(25, 3, 16).unfold(0, 10, 5).permute(0, 1, 3, 2)
    assert _dense_like(windows).stride() == (480, 16, 48, 1) and _dense_like(windows).shape == (4, 3, 10, 16)
    shared = torch.zeros(2, 10, 32).unfold(2, 16, 8).transpose(1, 2)
    assert _dense_like(shared).stride() == (480, 16, 48, 1)
    heads_last = torch.zeros(10, 2, 3, 48).permute(1, 2, 0, 3)[..., :16]
    assert _dense_like(heads_last).stride() == (48, 16, 96, 1)
    for view in (x[:, :1].expand(2, 3, 10, 16), x[:1, :1].expand(2, 3, 10, 16), x[..., :1, :].expand(2, 3, 10, 16), torch.zeros(2, 3, 16, 1).mT):
        made = _dense_like(view)
        assert made.shape == view.shape and made.stride(3) == 1 and made.untyped_storage().nbytes() == made.numel() * 4


def test_version_tells_the_descriptors_apart(lib):  # noqa: F811
    """The gradients' strides and `clear` lie behind what the descriptor of version 100 had, 128 bytes."""
    from paper_2507_08637_amd.binding import WersaDecayDesc
    assert lib.wersa_version() >= 200
    assert WersaDecayDesc.stride_dq.offset == 128 and WersaDecayDesc.clear.offset == 200 and ctypes.sizeof(WersaDecayDesc) == 208
