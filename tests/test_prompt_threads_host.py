"""Calls on any thread and stream right behind a layer's construction.  Threads that make the first prompt calls at once share one
description of its weights: a second one that replaced the first would give the first one's table back to the pool while kernels
still read tensor maps in it.  And the constructor returns when what it puts on the device is there.  Descriptions and
devices are stand-ins here, so no GPU is needed."""
import threading
import time

import numpy as np
import pytest

from paper_2601_21198_b200 import build


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def layer_of(zb, monkeypatch):
    """A layer of two experts whose constructor's GPU part is left out."""
    import torch
    hidden, inter = 8, 16
    monkeypatch.setattr(zb, "_get_kinds", lambda: type("Kinds", (), {"bf16": (torch.bfloat16,)}))
    monkeypatch.setattr(zb, "_device_of", lambda name, t: 0)
    monkeypatch.setattr(zb, "_dense", lambda name, t, shape, kinds, index: t.data_ptr())
    monkeypatch.setattr(zb, "_on_device", lambda index: torch.inference_mode())
    monkeypatch.setattr(zb, "zipmoe_resident_experts_plan", lambda *sizes: (np.zeros(64, np.uint8), zb.ResidentExpertsStruct()))
    monkeypatch.setattr(zb, "_scratch_of", lambda device, index: None)
    return zb.ResidentExperts([torch.zeros(hidden * inter, dtype=torch.bfloat16) for _ in range(6)], hidden, inter)


def test_one_description_for_all_threads(zb, monkeypatch):
    layer, made = layer_of(zb, monkeypatch), []

    class Slow:
        def __init__(self, matrices, up=None, status=None):
            assert status is layer.status and len(matrices) == 2
            time.sleep(0.05)
            made.append(self)

    monkeypatch.setattr(zb, "GroupedMatrix", Slow)
    start, got = threading.Barrier(4), []

    def first_call():
        start.wait()
        got.append(layer._products())

    threads = [threading.Thread(target=first_call) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 2 and all(g is got[0] for g in got) and layer._products() is got[0]


def test_the_status_is_zeroed_before_the_first_call(zb, monkeypatch):
    """On another stream a call could otherwise report an error that the zeroing then clears.  The copy of the table from the host
    returns when it and all before it on the stream is done, so it has to come last."""
    import torch
    steps, zeros, from_numpy = [], torch.zeros, torch.from_numpy

    class Table:
        def __init__(self, array):
            self.array = array

        def to(self, device):
            steps.append("copy")
            return from_numpy(self.array)

    monkeypatch.setattr(torch, "from_numpy", Table)
    monkeypatch.setattr(torch, "zeros", lambda *size, **kw: steps.append("zeros") or zeros(*size, **kw))
    layer_of(zb, monkeypatch)
    assert "zeros" in steps and steps[-1] == "copy"
