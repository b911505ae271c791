"""The workspaces of the tree calls are on the device of the other tensors: one elsewhere is
refused before the library is called (no GPU: the tensors only say where they are)."""
import types

import pytest
import torch

from paper_2606_31160_gb300 import sd


class _On(torch.Tensor):
    """A CPU tensor that says it is on a CUDA device."""

    at = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.at))

    def get_device(self):
        return self.at


def _on(at, *shape, dtype=torch.int32):
    t = torch.zeros(shape, dtype=dtype).as_subclass(_On)
    t.at = at
    return t


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library."""
    made = []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: made.append(name) or 0

    monkeypatch.setattr(sd, "lib", Lib)
    monkeypatch.setattr(sd, "_stream_on", lambda index: 0)
    return made


def _attend(ws_at):
    cache = types.SimpleNamespace(_shape=(2, 2, 128, 64), _device=0, _ref=None)
    q = _on(0, 2, 3, 4, 64, dtype=torch.bfloat16)
    return sd.tree_attention(q, cache, out=_on(0, 2, 3, 4, 64, dtype=torch.bfloat16), ws=_on(ws_at, 4096, dtype=torch.uint8))


def _accept(ws_at):
    ints = [_on(0, 2, 3) for _ in range(4)]
    return sd.accept_tree(_on(0, 2, 3, 50, dtype=torch.float32), ints[0], n_emit=_on(0, 2), path=ints[1], out=ints[2],
                          argmax=ints[3], ws=_on(ws_at, 4096, dtype=torch.uint8))


@pytest.mark.parametrize("call,name", [(_attend, "sd_tree_attention"), (_accept, "sd_accept_tree")])
def test_a_workspace_of_another_device_is_refused(calls, call, name):
    call(0)
    assert calls == [name]
    with pytest.raises(ValueError):
        call(1)
    assert calls == [name]
