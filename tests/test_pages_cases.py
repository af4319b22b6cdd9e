"""The timed cases of the page operators (CPU): each call is made on the stream that is current then."""
import importlib.util
import os

import pytest
import torch

tadm = pytest.importorskip("paper_2609_37924_amd")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def cases():
    spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(ROOT, "perf", "operators.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_calls_follow_the_current_stream(monkeypatch):
    """One handle per head layout, its stream set where the current one is another."""
    mod, made, streams, now = cases(), [], [], [11]
    monkeypatch.setattr(tadm, "tadm_model_create", lambda cfg: made.append(cfg) or len(made))
    monkeypatch.setattr(tadm, "tadm_set_stream", lambda m, s: streams.append((m, s)))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: now[0], raising=False)
    block, small = (dict(case=next(c for c in mod.listed() if c["heads"] == h), data=torch.zeros(1)) for h in (16, 12))
    for now[0], state, m in ((11, block, 1), (11, block, 1), (12, block, 1), (12, small, 2), (13, block, 1), (11, block, 1)):
        assert mod._handle(state)[1] == m
    assert len(made) == 2 and streams == [(1, 11), (1, 12), (2, 12), (1, 13), (1, 11)]
