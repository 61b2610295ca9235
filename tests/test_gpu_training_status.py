"""The example takes no step on gradients of a kernel that gave up a wait (stood in for by a failing status call)."""
import os
import sys

import pytest
import torch

import paper_2406_17918_b200 as gs

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_no_step_behind_a_failure(monkeypatch):
    import train_context_nodes as example

    asked, stepped = [], []

    def status(stream=None):
        asked.append(1)
        if len(asked) == 3:
            raise gs.GsError(6, "a kernel gave up")

    adam = torch.optim.Adam
    monkeypatch.setattr(example.gs, "gs_train_status", status)
    monkeypatch.setattr(example.torch.optim, "Adam", type("Adam", (adam,), {"step": lambda self, *a: (stepped.append(1), adam.step(self, *a))[1]}))
    with pytest.raises(gs.GsError):
        example.train("tiny", steps=10, log=lambda *a: None)
    assert len(stepped) == 2
