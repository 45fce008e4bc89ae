"""On which device the calls of the 8-bit cache go out, where it is not the
current one (no GPU: the calls themselves are stood in for)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2608_06557_amd import device

CLASSES = [device.DeviceKvAppend, device.DeviceAttention, device.DeviceSharedAttention, device.DeviceKvBounds,
           device.DeviceKvSelect, device.DeviceSelectedAttention, device.DeviceKvEvict]


@pytest.mark.parametrize("cls", CLASSES, ids=lambda c: c.__name__)
@pytest.mark.parametrize("where", [0, 3])
def test_calls_go_to_the_tensors_device(monkeypatch, cls, where):
    now, seen = [0], []

    class On:
        def __init__(self, d):
            self.to = torch.device(d).index

        def __enter__(self):
            self.was, now[0] = now[0], self.to

        def __exit__(self, *a):
            now[0] = self.was

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(device, "stream_handle", lambda stream=None: ("stream of", now[0]) if stream is None else stream)
    op, at = cls.__new__(cls), torch.device("cuda", where)
    op.kv = SimpleNamespace(pool=SimpleNamespace(device=at))
    op.status = SimpleNamespace(device=at)
    op._call = lambda stream: seen.append((now[0], stream)) or 0
    op.run()
    op.run("one of its own")
    assert seen == [(where, ("stream of", where)), (where, "one of its own")] and now == [0]
    op._call = lambda stream: -1
    with pytest.raises(Exception):
        op.run()
    assert now == [0]
