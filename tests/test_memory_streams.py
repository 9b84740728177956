"""CPU tests of the streams that the long-memory operators work on: which
stream's memory the binding takes, with torch's streams and the library replaced
by records of what was asked of them."""
import contextlib

import pytest
import torch

from paper_2607_20293_amd import evo


class _Stream:
    def __init__(self, handle, device=torch.device("cpu")):
        self.cuda_stream, self.device = handle, device


class _Record:
    """What happened, in order: (what, stream handle)."""

    def __init__(self, monkeypatch):
        self.current, self.made, self.launched, self.kept = _Stream(7), [], [], []
        new_empty = torch.Tensor.new_empty

        def made(t, *a, **kw):
            out = new_empty(t, *a, **kw)
            self.made.append((self.current.cuda_stream, out.data_ptr()))
            return out

        @contextlib.contextmanager
        def entered(stream):
            before, self.current = self.current, stream
            yield
            self.current = before
        monkeypatch.setattr(torch.Tensor, "new_empty", made)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.kept.append((t.data_ptr(), s.cuda_stream)))
        monkeypatch.setattr(torch.cuda, "stream", entered)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(evo, "_current_stream", lambda index: self.current.cuda_stream)
        monkeypatch.setattr(evo, "_current_device", lambda: None)
        monkeypatch.setattr(evo, "_device_of", lambda t: t.device)
        monkeypatch.setattr(evo, "lib", lambda: self)

    def __getattr__(self, name):
        if not name.startswith("evo_"):
            raise AttributeError(name)
        if name == "evo_chunk_attention_workspace":
            return lambda *a: 4096

        def call(*args):
            self.launched.append((name, args[-1]))
            return 0
        return call


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def _calls():
    cache = evo.KVCache(torch.zeros(2, 2, 64, 32, dtype=torch.int8), torch.zeros(2, 2, 32, 64, dtype=torch.int8),
                        torch.zeros(2, 2, 64), torch.zeros(2, 2, 64))
    q, k = torch.zeros(3, 4, 32), torch.zeros(3, 2, 32)
    tab, one, pos, rope = _ints(0, 1)[None], _ints(3), _ints(0, 1, 2), torch.zeros(9, 16, 2)
    gain = torch.ones(32)
    return [
        ([q, k, pos, rope, gain], 2, lambda **kw: evo.qk_norm_rope(q, k, pos, rope, gain, gain, **kw)),
        ([*(t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), tab, one, k], 0, lambda **kw: evo.cache_write(cache, tab, one, k, k, **kw) or ()),
        ([*(t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), tab, one], 2, lambda **kw: evo.cache_read(cache, tab, one, 3, torch.float32, **kw)),
        ([*(t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), tab, one, q, k, rope], 1, lambda **kw: (evo.qkv_write(cache, tab, one, q, k, k, rope, **kw),)),
        ([*(t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), tab, one, q], 2, lambda **kw: evo.chunk_attention(q, cache, tab, one, prefix=one, **kw))]


@pytest.mark.parametrize("i", range(5))
def test_what_a_call_makes_belongs_to_its_stream(monkeypatch, i):
    """A block of the current stream's pool may still be in use there: outputs
    and workspaces of a call on another stream come from that stream's."""
    rec = _Record(monkeypatch)
    given, n_out, call = _calls()[i]
    side = _Stream(11)
    outs = call(stream=side)
    assert rec.launched and all(h == 11 for _, h in rec.launched)
    assert len(rec.made) >= n_out and all(h == 11 for h, _ in rec.made)
    assert rec.current.cuda_stream == 7
    # what was given stays until the side stream's work is done, what is returned
    # until the caller's
    for t in given:
        assert (t.data_ptr(), 11) in rec.kept
    assert len(outs) == n_out and all((t.data_ptr(), 7) in rec.kept for t in outs)


@pytest.mark.parametrize("i", range(5))
def test_calls_on_the_current_stream(monkeypatch, i):
    rec = _Record(monkeypatch)
    _, _, call = _calls()[i]
    for kw in ({}, dict(stream=_Stream(7))):
        del rec.made[:], rec.launched[:]
        call(**kw)
        assert all(h == 7 for _, h in rec.launched) and all(h == 7 for h, _ in rec.made) and not rec.kept


def test_a_stream_of_another_device_is_refused(monkeypatch):
    rec = _Record(monkeypatch)
    for _, _, call in _calls():
        with pytest.raises(ValueError, match="stream"):
            call(stream=_Stream(11, torch.device("cuda", 1)))
    assert not rec.launched
