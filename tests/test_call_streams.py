"""What the operators on caller-held caches do with the tensors of a call on another stream.  No device: the stream is a stand-in."""
import contextlib

import pytest
import torch

import paper_2502_07861_b200.binding as binding


class _Stream:
    cuda_stream = 5


class _External(_Stream):
    """A stream that somebody else made, and may have destroyed when a tensor's memory is freed."""

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def recorded(monkeypatch):
    seen = []
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "ExternalStream", _External)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: seen.append((t, stream)))
    return seen


def _launches_nothing(monkeypatch):
    """The calls' own work replaced: none of their tensors is on a device."""
    class Lib:
        def __getattr__(self, name):
            return lambda *args: 0

    monkeypatch.setattr(binding, "load", lambda: Lib())
    monkeypatch.setattr(binding, "_on_current", lambda *args: None)
    monkeypatch.setattr(binding, "_workspace_bytes", lambda *args: 0)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)


def _calls():
    k, v, q, score, pos, lens = torch.zeros(2, 9, 64), torch.zeros(2, 9, 64), torch.zeros(2, 3, 64), torch.zeros(2, 9), torch.zeros(2, 9, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    out = {"k": torch.zeros(2, 4, 64), "v": torch.zeros(2, 4, 64), "score": torch.zeros(2, 4)}
    k4, v4, q3, w, oq, os = torch.zeros(5, 2, 7, 64), torch.zeros(5, 2, 7, 64), torch.zeros(5, 6, 64), torch.ones(2, 9), torch.zeros(2, 3, 64), torch.zeros(2, 9)
    lens5 = torch.ones(5, dtype=torch.int32)
    return [
        (lambda stream: binding.attn_scored(k, v, q, lens=lens, score=score, score_out=os, out=oq, stream=stream), [k, v, q, lens, score, os, oq]),
        (lambda stream: binding.cache_evict(k, v, score, 4, lens=lens, pos=pos, out=out, stream=stream), [k, v, score, lens, pos, *out.values()]),
        (lambda stream: binding.cache_evict(k, v, score, 4, lens=lens, pos=pos, in_place=True, stream=stream), [k, v, score, lens, pos]),
        (lambda stream: binding.decode_attn_prefix(k, v, k4, v4, q3, lens=lens5, weight=w, stream=stream), [k, v, k4, v4, q3, lens5, w]),
    ]


@pytest.mark.parametrize("which", range(4))
def test_tensors_given_are_recorded_on_the_stream(monkeypatch, recorded, which):
    """The allocator may hand a temporary's memory on as soon as the caller lets it go, unless it knows of the other stream."""
    _launches_nothing(monkeypatch)
    call, tensors = _calls()[which]
    stream = _Stream()
    call(stream)
    for t in tensors:
        assert any(t is r and s is stream for r, s in recorded)


@pytest.mark.parametrize("which", range(4))
def test_nothing_is_recorded_on_a_raw_stream_or_the_current_one(monkeypatch, recorded, which):
    _launches_nothing(monkeypatch)
    call, _ = _calls()[which]
    call(5)
    call(_External(5))
    call(None)
    assert not recorded
