"""A stage's exported keys and values belong to the current stream, on whichever stream the stage works: the order of waits, without a device."""
import types

import pytest
import torch

from paper_2511_14450_amd import binding


class Stream:
    def __init__(self, name, handle, log):
        self.name, self.cuda_stream, self.log = name, handle, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


@pytest.mark.parametrize("aside", [False, True])
def test_an_export_is_ordered_with_the_current_stream(monkeypatch, aside):
    log = []
    here, there = Stream("here", 0, log), Stream("there", 7, log)

    class Library:
        def stage_context_len(self, handle, request, out):
            out._obj.value = 5
            return binding.HYP_OK

        def stage_export_kv(self, handle, layer, request, k, v):
            log.append("export")
            return binding.HYP_OK

    empty = torch.empty
    monkeypatch.setattr(binding, "load_library", lambda: Library())
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: empty(shape, dtype=dtype))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *device: here)
    cfg = types.SimpleNamespace(n_kv_heads=2, head_dim=4, dtype=binding.HYP_F32)
    stage = types.SimpleNamespace(handle=1, cfg=cfg, stream=there if aside else Stream("here", 0, log))
    k, v = binding.stage_export_kv(stage, 0, 0)
    assert k.shape == v.shape == (5, 8)
    assert log == ([("there", "waits for", "here"), "export", ("here", "waits for", "there")] if aside else ["export"])
