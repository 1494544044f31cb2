"""On which device and stream the operators' calls run (host logic: stand-ins for tensors, streams and
the library's functions, nothing is launched)."""
import contextlib

import pytest
import torch

from paper_1712_01887_b200 import binding as B


class Tensor:
    """What the binding asks of a tensor; its memory is not there."""

    def __init__(self, shape, dtype=torch.float32, device=1):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device

    def get_device(self):
        return self.device

    def stride(self):
        return tuple(int(torch.Size(self.shape[i + 1:]).numel()) for i in range(len(self.shape)))

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()


class Stream:
    def __init__(self, handle, device_index):
        self.cuda_stream, self.device_index = handle, device_index


@pytest.fixture
def machine(monkeypatch):
    """Two devices, device 0 current; `calls`: (device that was current, stream) of every call made."""
    m = type("Machine", (), {"current": 0, "calls": []})()

    @contextlib.contextmanager
    def device(d):
        before, m.current = m.current, d
        try:
            yield
        finally:
            m.current = before

    def called(args, stream):
        m.calls.append((m.current, stream))
        return 0

    monkeypatch.setattr(B, "_current_device", lambda: m.current, raising=False)
    monkeypatch.setattr(B, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    for name in ("dgc_top_logits", "dgc_gated_scan_step", "dgc_gated_scan_forward", "dgc_gated_scan_backward", "dgc_distill_forward",
                 "dgc_distill_backward", "dgc_distill_loss_grad"):
        monkeypatch.setattr(B._lib, name, called)
    return m


def _all_calls(device, **how):
    m = lambda: Tensor((6, 40), device=device)  # noqa: E731
    v = lambda *s: Tensor(s, device=device)     # noqa: E731
    i = Tensor((6, 3), torch.int32, device)
    yield lambda: B.top_logits(m(), i, v(6, 3), **how)
    yield lambda: B.gated_scan_step(m(), m(), v(6, 40), m(), **how)
    yield lambda: B.gated_scan_forward(m(), m(), m(), **how)
    yield lambda: B.gated_scan_backward(m(), m(), m(), m(), m(), m(), **how)
    yield lambda: B.distill_forward(m(), i, v(6, 3), v(6), v(6, 2), **how)
    yield lambda: B.distill_backward(m(), i, v(6, 3), v(6, 2), v(6), m(), **how)
    yield lambda: B.distill_loss_grad(m(), i, v(6, 3), v(6), v(6), m(), **how)


@pytest.mark.parametrize("device", [0, 1])
def test_calls_run_on_the_tensors_device(machine, device):
    """The current device need not be the tensors': a call makes theirs current, and puts it back."""
    for call in _all_calls(device):
        call()
    assert machine.calls == [(device, 100 + device)] * 7 and machine.current == 0


def test_a_given_stream_is_of_the_tensors_device(machine):
    for call in _all_calls(1, stream=Stream(77, 1)):
        call()
    for call in _all_calls(1, stream=55):
        call()
    assert machine.calls == [(1, 77)] * 7 + [(1, 55)] * 7
    for call in _all_calls(1, stream=Stream(0, 0)):   # the default stream of another device
        with pytest.raises(ValueError):
            call()
    assert len(machine.calls) == 14 and machine.current == 0


def test_the_workspace_comes_from_the_calls_stream(machine, monkeypatch):
    """Torch's allocator is asked on the very stream that the kernels run on, the default stream's
    handle 0 included (an external stream of handle 0 is one of torch's own streams)."""
    now, asked = [None], []

    @contextlib.contextmanager
    def stream(s):
        before, now[0] = now[0], s.cuda_stream
        try:
            yield
        finally:
            now[0] = before

    def empty(n, **how):
        asked.append((n, now[0], how["device"]))
        return Tensor((n,), torch.uint8, 1)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: Stream(handle or "a stream of torch's", device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: Stream(0, device))
    monkeypatch.setattr(torch, "empty", empty)
    m = [Tensor((8192, 40)) for _ in range(6)]
    need = (8192 // 64 + 1) * 40 * 8
    for given, handle in ((None, None), (Stream(77, 1), 77), (Stream(0, 1), 0), (55, 55), (0, 0)):
        asked.clear()
        B.gated_scan_forward(*m[:3], stream=given)
        B.gated_scan_backward(*m, stream=given)
        assert asked == [(need, handle, "cuda:1")] * 2 and now[0] is None
        assert machine.calls[-2:] == [(1, 101 if given is None else handle)] * 2
