"""Workspaces: sizes that the binding keeps hold for the device they were asked for, and what is handed
over as one is device memory in one piece."""

import pytest
import torch


def test_sizes_are_kept_for_each_device(monkeypatch):
    from paper_2608_03020_gb300 import loca

    device, asked = [0], []

    class Lib:
        def __getattr__(self, name):
            def size(*args):
                asked.append((device[0], name, args[:-1]))
                args[-1]._obj.value = 1000 * (device[0] + 1) + args[0]
                return 0

            return size

    monkeypatch.setattr(loca, "lib", lambda: Lib())
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device[0])
    calls = [lambda: loca.head_loss_workspace_size(123457, 11, 8, 1),
             lambda: loca.head_loss_backward_workspace_size(123457, 11, 8, True, False),
             lambda: loca.adapter_workspace_size(123457, 8, 8, 3, 2, backward=True)]
    for call in calls:
        asked.clear()
        for device[0] in (0, 1, 0, 1):
            assert call() == 1000 * (device[0] + 1) + 123457
        assert len(asked) == 2 and asked[0][1] == asked[1][1]
    loca._size_on.cache_clear()  # (what this stand-in said)


def test_a_workspace_in_host_memory_is_refused():
    from paper_2608_03020_gb300 import loca

    with pytest.raises(TypeError):
        loca._workspace(64, "cuda", torch.empty(64, dtype=torch.uint8))
    with pytest.raises(TypeError):
        loca._workspace(64, "cuda", bytearray(64))
