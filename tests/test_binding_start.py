"""The first serving call of a process, made by two threads at once."""
import sys
import types

import torch

import paper_2502_01681_amd as dg4
from paper_2502_01681_amd import binding


def test_a_first_call_while_another_one_is_being_set_up(monkeypatch):
    """The second call comes at every point of the first one's set-up in turn: whenever torch is asked for something."""
    cfg = dg4.LayerConfig(128, 4, 2, 1, "bf16")
    tensor = types.SimpleNamespace(get_device=lambda: 0)
    asked = {"_cuda_getCurrentRawStream": lambda dev: 77, "_cuda_getDevice": lambda: 0}
    for point in range(8):
        seen = []

        class Torch:
            def __getattr__(self, name):
                seen.append(name)
                if len(seen) - 1 == point:         # (what the second call asks for comes behind this)
                    assert binding._call("second", cfg, tensor) == (torch.bfloat16, 0, 77)
                if name == "_C":
                    return types.SimpleNamespace(**asked)
                return getattr(torch, name)

        with monkeypatch.context() as m:
            m.setitem(sys.modules, "torch", Torch())
            m.setattr(binding, "_types", None)
            for name in ("_raw_stream", "_device"):
                m.delattr(binding, name, raising=False)
            assert binding._call("first", cfg, tensor) == (torch.bfloat16, 0, 77)
            for name in ("_raw_stream", "_device"):            # (as found: set by the first call of a process)
                delattr(binding, name)
        assert len(seen) > min(point, 5)
