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
    """One handle per head layout, its stream set anew by every call."""
    mod, made, streams = cases(), [], []

    class Stream:
        cuda_stream = 11

    monkeypatch.setattr(tadm, "tadm_model_create", lambda cfg: made.append(cfg) or len(made))
    monkeypatch.setattr(tadm, "tadm_set_stream", lambda m, s: streams.append((m, s)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream)
    block, small = (dict(case=next(c for c in mod.listed() if c["heads"] == h)) for h in (16, 12))
    assert mod._handle(block)[1] == 1
    Stream.cuda_stream = 12
    assert mod._handle(block)[1] == 1 and mod._handle(small)[1] == 2
    Stream.cuda_stream = 13
    assert mod._handle(block)[1] == 1
    assert len(made) == 2 and streams == [(1, 11), (1, 12), (2, 12), (1, 13)]
