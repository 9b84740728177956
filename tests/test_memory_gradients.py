"""CPU tests: the long-memory operators refuse tensors whose gradient they would
lose (their arguments are checked before the library is called)."""
import pytest
import torch

from paper_2607_20293_amd import evo


class _Library:
    """Takes every call and counts them."""
    calls = 0

    def __getattr__(self, name):
        if name == "evo_chunk_attention_workspace":
            return lambda *a: 0

        def call(*a):
            self.calls += 1
            return 0
        return call


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def _cases():
    """(name of the tensor that requires a gradient, call with the tensors)."""
    cache = evo.KVCache(torch.zeros(2, 2, 64, 32), torch.zeros(2, 2, 32, 64))
    tab, one, pos = _ints(0, 1)[None], _ints(3), _ints(0, 1, 2)

    def rope(q, k, table, q_gain, k_gain, out):
        return evo.qk_norm_rope(q, k, pos, table, q_gain, k_gain, out=(out, torch.zeros(3, 2, 32)))

    def write(k, v):
        return evo.cache_write(cache, tab, one, k, v)

    def fused(q, k, v, table, q_gain, k_gain):
        return evo.qkv_write(cache, tab, one, q, k, v, table, q_gain, k_gain)

    def attend(q, slopes, lse):
        return evo.chunk_attention(q, cache, tab, one, slopes=slopes, lse=lse)

    def held(k, v):
        return evo.KVCache(k, v)
    shapes = dict(q=(3, 4, 32), k=(3, 2, 32), v=(3, 2, 32), table=(9, 16, 2), q_gain=(32,), k_gain=(32,), out=(3, 4, 32),
                  slopes=(4,), lse=(3, 4))
    for f in (rope, write, fused, attend, held):
        names = f.__code__.co_varnames[:f.__code__.co_argcount]
        for name in names:
            sizes = {**shapes, "k": (2, 2, 64, 32), "v": (2, 2, 32, 64)} if f is held else shapes
            yield f.__name__, name, f, {n: sizes[n] for n in names}


def test_tensors_that_require_a_gradient_are_refused(monkeypatch):
    library = _Library()
    monkeypatch.setattr(evo, "lib", lambda: library)
    monkeypatch.setattr(evo, "_device_of", lambda t: t.device)
    monkeypatch.setattr(evo, "_current_device", lambda: None)
    monkeypatch.setattr(evo, "_current_stream", lambda index: 0)
    for what, name, f, sizes in _cases():
        t = {n: torch.zeros(s) for n, s in sizes.items()}
        t[name].requires_grad_(True)
        before = library.calls
        with pytest.raises(RuntimeError, match=name + ".*gradient"):
            f(**t)
        assert library.calls == before, (what, name)
        # nothing is lost where no gradient is recorded, or of detached tensors
        with torch.no_grad():
            f(**t)
        f(**{n: x.detach() for n, x in t.items()})
        assert library.calls == before + (2 if what != "held" else 0), (what, name)
