"""Where the scratch memory of mx_rmsnorm_bwd lives (no GPU: the library's call is written down, not made, and torch's streams are stand-ins).

A tensor that is dropped when the call returns goes back to torch's allocator, which gives it to whoever asks next.  On torch's current stream that is in
order, since whoever asks next works behind the call.  A captured call runs again with every replay, so its scratch memory has to live as long as its results."""
import types

import pytest
import torch

from paper_2310_10537_amd import binding

CURRENT, OTHER = types.SimpleNamespace(cuda_stream=11), types.SimpleNamespace(cuda_stream=12)


@pytest.fixture
def call(monkeypatch):
    """mx_rmsnorm_bwd on host tensors; returns (dweight, address of the scratch memory or None, its size)."""
    captured = set()
    inside = [CURRENT.cuda_stream]

    class Entered:
        def __init__(self, to):
            self.to = to

        def __enter__(self):
            inside.append(getattr(self.to, "cuda_stream", inside[-1]))

        def __exit__(self, *_):
            inside.pop()

    monkeypatch.setattr(binding, "_where", lambda t, name: -1)
    monkeypatch.setattr(binding, "_dev", lambda t, name: None)
    monkeypatch.setattr(binding, "_made", lambda shape, dtype, index: torch.empty(shape, dtype=dtype))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: inside[-1], raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: inside[-1] in captured)
    monkeypatch.setattr(torch.cuda, "device", lambda index: Entered(None))
    monkeypatch.setattr(torch.cuda, "stream", Entered)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: types.SimpleNamespace(cuda_stream=raw))
    seen = []
    monkeypatch.setattr(binding, "_call", lambda index, stream, fn, *args: seen.append(args))

    def run(rows, cols, stream=None, capture=(), **kw):
        captured.clear()
        captured.update(s.cuda_stream for s in capture)
        x = torch.zeros((rows, cols))
        dx, dw = binding.mx_rmsnorm_bwd(x, x, None, torch.ones((rows,)), stream=stream, **kw)
        *_, pointer, bytes_ = seen[-1]
        assert seen[-1][-3] == (None if dw is None else dw.data_ptr())
        return dw, pointer, bytes_
    return run


SIZES = [(1, 4), (333, 1000), (64, 516), (4096, 2048), (5, 20000)]


def whole(t):
    s = t.untyped_storage()
    return s.data_ptr(), s.data_ptr() + s.nbytes()


@pytest.mark.parametrize("rows,cols", SIZES, ids=str)
def test_captured_calls_keep_it_with_the_result(call, rows, cols):
    need = binding.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols)
    for kw in (dict(capture=(CURRENT,)), dict(capture=(CURRENT,), stream=CURRENT), dict(capture=(OTHER,), stream=OTHER), dict(capture=(CURRENT, OTHER), stream=OTHER)):
        dw, pointer, size = call(rows, cols, **kw)
        first, end = whole(dw)
        assert dw.shape == (cols,) and dw.dtype == torch.float32 and dw.is_contiguous() and dw.data_ptr() % 16 == 0
        assert pointer is not None and pointer % 16 == 0 and size >= need, kw
        assert dw.data_ptr() + 4 * cols <= pointer and first <= pointer and pointer + size <= end, kw


@pytest.mark.parametrize("rows,cols", SIZES, ids=str)
def test_other_calls_give_it_back(call, rows, cols):
    need = binding.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols)
    for kw in (dict(), dict(stream=CURRENT), dict(capture=(OTHER,))):
        dw, pointer, size = call(rows, cols, **kw)
        first, end = whole(dw)
        assert end - first == 4 * cols and pointer is not None and size >= need and not first <= pointer < end, kw
    for capture in ((), (CURRENT,)):                     # a stream that is neither the current one nor captured: the library's own, in that stream's order
        dw, pointer, size = call(rows, cols, stream=OTHER, capture=capture)
        assert pointer is None and size == 0 and whole(dw)[1] - whole(dw)[0] == 4 * cols


def test_none_without_a_weight_gradient_or_rows(call):
    for capture in ((), (CURRENT,)):
        assert call(100, 1000, want_dweight=False, capture=capture)[1:] == (None, 0)
        dw, pointer, size = call(0, 1000, capture=capture)
        assert dw.shape == (1000,) and pointer is None and size == 0


def test_the_null_stream_is_never_captured(call, monkeypatch):
    """(torch makes a stream of its own of a handle that is zero.)"""
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: OTHER)
    dw, pointer, size = call(333, 1000, stream=types.SimpleNamespace(cuda_stream=0), capture=(OTHER,))
    assert pointer is None and size == 0 and whole(dw)[1] - whole(dw)[0] == 4000
