"""When a BlockMask keeps its transpose and when it builds another, with stand-ins for the device: no GPU needed."""

import ctypes

import pytest

import paper_2505_22918_amd as rt


class _Device:
    """What the binding asks of the device: the current stream, whether it is captured, and the launches it was given."""

    def __init__(self):
        self.stream, self.capturing, self.idle = 1, False, False  # idle: all work has ended
        self.built, self.waits, self.held = [], [], []

    # the library
    def rt_index_transpose_size(self, mask, room, values):
        ctypes.cast(values, ctypes.POINTER(ctypes.c_int64))[0] = room + 64
        return 0

    def rt_index_transpose(self, mask, T, t, stream):
        self.built.append((stream, self.capturing))
        return 0


@pytest.fixture
def device(monkeypatch):
    import contextlib

    import torch

    dev = _Device()

    class Stream:
        def wait_event(self, event):
            dev.waits.append((dev.stream, event.at))

    class Event:
        def record(self, stream=None):
            self.at = dev.stream

        def query(self):
            return dev.idle

    monkeypatch.setattr(rt, "_stream", lambda t: dev.stream)
    monkeypatch.setattr(rt, "_on", lambda t: contextlib.nullcontext())
    monkeypatch.setattr(rt._lib, "load", lambda: dev)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: dev.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: dev.held.append(t.data_ptr()))
    return dev


def _mask():
    import torch

    return rt.BlockMask(torch.arange(5, dtype=torch.int32), torch.arange(4, dtype=torch.int32), 64, 4, 4)


def test_a_mask_of_many_steps_is_transposed_once(device):
    mask = _mask()
    t = mask.transposed()
    assert mask.transposed() is t and device.built == [(1, False)] and not device.waits


def test_another_stream_waits_and_holds_the_memory(device):
    mask = _mask()
    t = mask.transposed()
    device.stream = 2
    assert mask.transposed() is t and device.waits == [(2, 1)]
    assert set(device.held) == {t.row_ptr.data_ptr(), t.col_idx.data_ptr()}


def test_a_capture_builds_its_own(device):
    """A graph keeps the addresses that its capture saw, a mask may replace the transpose it keeps: what a capture uses
    is built by the graph, in the graph's memory."""
    mask = _mask()
    kept = mask.transposed()
    device.idle, device.stream = True, 2
    mask.transposed()
    for stream in (1, 2):
        device.stream, device.capturing = stream, True
        t = mask.transposed()
        assert t is not kept and t.col_idx.data_ptr() != kept.col_idx.data_ptr()
        assert device.built[-1] == (stream, True)
    device.stream, device.capturing = 1, False
    assert mask.transposed() is kept and len(device.built) == 3


def test_arrays_whose_writes_are_not_counted(device):
    """Inference tensors have no version: nothing is kept that a write could leave behind."""
    import torch

    with torch.inference_mode():
        mask = _mask()
    first = mask.transposed()
    with torch.inference_mode():
        mask.col_idx.add_(0)
    assert mask.transposed() is not first and len(device.built) == 2


def test_a_write_in_a_capture_counts_once_and_happens_at_every_replay(device):
    mask = _mask()
    mask.transposed()
    device.capturing = True
    mask.col_idx.add_(0)
    device.capturing = False
    seen = [mask.transposed() for _ in range(3)]
    assert len({id(t) for t in seen}) == 3 and len(device.built) == 4


@pytest.mark.parametrize("written", ["row_ptr", "col_idx"])
def test_arrays_written_before_the_mask_is_made(device, written):
    """Static buffers that a graph fills: the capture may have come first."""
    import torch

    arrays = {"row_ptr": torch.arange(5, dtype=torch.int32), "col_idx": torch.arange(4, dtype=torch.int32)}
    arrays[written].copy_(arrays[written].clone())
    mask = rt.BlockMask(arrays["row_ptr"], arrays["col_idx"], 64, 4, 4)
    assert mask.transposed() is not mask.transposed()


def test_a_mask_made_under_a_capture(device, monkeypatch):
    """By the framework or by hand."""
    import torch

    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    device.capturing = True
    mask = _mask()
    device.capturing = False
    assert mask.transposed() is not mask.transposed()
    assert _mask().transposed() is not None


def test_anew_replaces_the_kept_one(device):
    mask = _mask()
    first = mask.transposed()
    second = mask.transposed(anew=True)
    assert second is not first and mask.transposed() is second and len(device.built) == 2


def test_a_mask_restored_from_its_fields_alone(device):
    """As copies of masks that were stored earlier come back: without what their making notes."""
    whole = _mask()
    mask = object.__new__(rt.BlockMask)
    mask.__dict__.update({f: getattr(whole, f) for f in rt.BlockMask.__dataclass_fields__})
    assert mask.transposed() is mask.transposed()
