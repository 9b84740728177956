"""CPU tests: the operators over long memories and of the layers around their
attention refuse tensors with a tangent, which they would lose (arguments are checked
before the library is called)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2607_20293_amd import evo
from tests.test_memory_gradients import _cases, _Library


@pytest.fixture
def library(monkeypatch):
    made = _Library()
    monkeypatch.setattr(evo, "lib", lambda: made)
    monkeypatch.setattr(evo, "_device_of", lambda t: t.device)
    monkeypatch.setattr(evo, "_current_device", lambda: None)
    monkeypatch.setattr(evo, "_current_stream", lambda index: 0)
    return made


def _layer_cases():
    w = evo.Weights4(torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8), 32)

    def linear(x, bias, out):
        return evo.linear4(x, w, bias, out=out)

    def norm(x, y, gate, scale, shift, pre_gain, pre_bias, post_gain, post_bias, x_out, h_out):
        return evo.block_norm(x, y, post="rms", pre_gain=pre_gain, pre_bias=pre_bias, post_gain=post_gain, post_bias=post_bias,
                              gate=gate, scale=scale, shift=shift, x_out=x_out, h_out=h_out)
    shapes = dict(x=(6, 32), y=(6, 32), gate=(2, 32), scale=(2, 32), shift=(2, 32), pre_gain=(32,), pre_bias=(32,),
                  post_gain=(32,), post_bias=(32,), x_out=(6, 32), h_out=(6, 32), bias=(8,), out=(6, 8))
    for f in (linear, norm):
        names = f.__code__.co_varnames[:f.__code__.co_argcount]
        for name in names:
            yield f.__name__, name, f, {n: shapes[n] for n in names}


def test_tensors_with_a_tangent_are_refused(library):
    for what, name, f, sizes in [*_cases(), *_layer_cases()]:
        t = {n: torch.zeros(s) for n, s in sizes.items()}
        with forward_ad.dual_level():
            f(**t)                                                  # plain tensors within a level
            t[name] = forward_ad.make_dual(t[name], torch.ones_like(t[name]))
            before = library.calls
            # (tangents are passed on under no_grad too)
            for mode in (torch.enable_grad(), torch.no_grad()):
                with mode, pytest.raises(RuntimeError, match=name + ".*tangent"):
                    f(**t)
            assert library.calls == before, (what, name)
            f(**{n: x.detach() for n, x in t.items()})
            with torch.inference_mode():
                f(**t)
            assert library.calls == before + (2 if what != "held" else 0), (what, name)
        f(**t)                                                      # the level has ended, and the tangent with it


def test_views_and_matrices_with_a_tangent(library):
    w = evo.Weights4(torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8), 32)
    with forward_ad.dual_level():
        x = forward_ad.make_dual(torch.zeros(6, 64), torch.ones(6, 64))
        with pytest.raises(RuntimeError, match="x.*tangent"):
            evo.linear4(x[:, 32:], w)
    assert not library.calls
