"""What the binding of the operators around the pass refuses or falls back to, without a GPU."""
import pytest
import torch

from paper_2608_27128_gb300 import twinkv as tk


class OnDevice(torch.Tensor):
    """A tensor of the CPU that says it is on a CUDA device: the checks read no memory."""

    def get_device(self):
        return 0

    @property
    def device(self):
        return torch.device("cuda", 0)


def on_device(t):
    return t.as_subclass(OnDevice)


def workspaces(n):
    one = torch.zeros(1, dtype=torch.uint8)
    wide = torch.zeros(2 * n, dtype=torch.uint8)
    return [one.expand(n), wide[::2], wide.view(2, n)[:, :n // 2].expand(2, n // 2)]


def test_a_workspace_that_is_not_contiguous_is_refused():
    """It has as many elements as are asked for, and not that many bytes from its address on."""
    n = 4096
    assert tk._bytes(on_device(torch.zeros(n, dtype=torch.uint8)), n, 0, None).numel() == n
    for ws in workspaces(n):
        if ws.is_contiguous():
            continue
        assert ws.numel() >= n
        with pytest.raises(ValueError):
            tk._bytes(on_device(ws), n, 0, None)


def test_a_workspace_of_the_pass_has_to_be_contiguous_and_on_the_device():
    s = tk.Shape(1, 2, 600, 128, tk.BF16)
    n = tk.twinkv_workspace_size(s, tk.OP_REPAIR)
    dev = torch.device("cuda", 0)
    assert tk._ws(on_device(torch.zeros(n, dtype=torch.uint8)), s, tk.OP_REPAIR, dev).numel() == n
    for ws in workspaces(n):
        if ws.is_contiguous():
            continue
        with pytest.raises(ValueError):
            tk._ws(on_device(ws), s, tk.OP_REPAIR, dev)
    with pytest.raises(ValueError):
        tk._ws(torch.zeros(n, dtype=torch.uint8), s, tk.OP_REPAIR, dev)


@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32 + 1, 2.5, "7"])
def test_windows_and_sinks_beyond_32_bits_are_refused(value):
    """ctypes would take them modulo 2^32: a window of 2^32 + 5 as one of 5."""
    with pytest.raises((ValueError, TypeError)):
        tk._int32(value, "window")


def test_windows_and_sinks_of_32_bits():
    import numpy as np
    for value in (0, 4, 2 ** 31 - 1, -1, np.int64(300), True):
        assert tk._int32(value, "window") == value


def test_current_stream_without_torchs_private_calls(monkeypatch):
    """A torch that lacks the calls beneath torch.cuda's gets the public ones."""
    class Bare:
        pass

    class Stream:
        cuda_stream = 4711

    monkeypatch.setattr(torch, "_C", Bare())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: Stream())
    device, raw = tk._current_calls()
    assert device() == 3 and raw(3) == 4711
