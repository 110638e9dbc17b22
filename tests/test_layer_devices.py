"""The calls of rotary.py and chunk.py take tensors of the current GPU only (CPU)."""
import types

import pytest
import torch

from paper_2510_26577_amd import cache4, chunk, rotary
from tests import test_layer_arguments as arguments


@pytest.mark.parametrize("device,current,right", [("cuda:0", 0, True), ("cuda:1", 1, True), ("cuda:1", 0, False), ("cuda:0", 1, False)])
def test_tensors_of_another_gpu_are_refused(monkeypatch, device, current, right):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    t = types.SimpleNamespace(is_cuda=True, device=torch.device(device))
    if right:
        cache4._on_current_gpu(t)
    else:
        with pytest.raises(ValueError, match="current GPU"):
            cache4._on_current_gpu(t)


@pytest.mark.parametrize("which", list(arguments.MAKE))
def test_every_call_asks(monkeypatch, which):
    """(Host tensors that pass the checks of a call, up to this one.)"""
    asked = []

    def ask(t):
        asked.append(t)
        raise ValueError("asked")

    for module in (rotary, chunk):
        monkeypatch.setattr(module, "_on_current_gpu", ask)
    call = {"rotate": rotary.rotate, "append": rotary.append, "attn": lambda **kw: chunk.attn(kw.pop("q"), kw.pop("cache"), kw.pop("cu_T"), kw.pop("L"), **kw)}[which]
    with pytest.raises(ValueError, match="asked"):
        call(**arguments.MAKE[which][1]())
    assert len(asked) == 1
