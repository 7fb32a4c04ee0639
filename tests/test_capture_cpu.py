"""Whether a call that is not for captured streams asks about the stream of its tensors' device, whichever device is the current one."""
import contextlib

import pytest
import torch

from paper_1804_10727_amd import tokens


class OnTheGpu:
    is_cuda = True

    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.mark.parametrize("current,mine,captured,refused", [(0, 0, 0, True), (0, 1, 1, True), (0, 1, 0, False), (1, 0, 1, False), (1, 0, 0, True), (0, 0, None, False)])
def test_the_tensors_device_is_asked(monkeypatch, current, mine, captured, refused):
    now = [torch.device("cuda", current)]

    @contextlib.contextmanager
    def device(d):
        now.append(d)
        yield
        now.pop()
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now[-1].index == captured)
    with pytest.raises(RuntimeError, match="captured") if refused else contextlib.nullcontext():
        tokens._no_capture(OnTheGpu(mine))
    tokens._no_capture(torch.zeros(1))
