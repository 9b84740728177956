"""CPU tests: tensors that a caller hands an operator to write into are kept until the
work of the stream that it runs on is done, as its other tensors are."""
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.test_memory_streams import _ints, _Record, _Stream


def _calls():
    cache = evo.KVCache(torch.zeros(2, 2, 64, 32, dtype=torch.int8), torch.zeros(2, 2, 32, 64, dtype=torch.int8),
                        torch.zeros(2, 2, 64), torch.zeros(2, 2, 64))
    q, k = torch.zeros(3, 4, 32), torch.zeros(3, 2, 32)
    tab, one, pos, rope = _ints(0, 1)[None], _ints(3), _ints(0, 1, 2), torch.zeros(9, 16, 2)
    w = evo.Weights4(torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8), 32)
    x = torch.zeros(3, 32)
    outs = [torch.zeros(3, 4, 32), torch.zeros(3, 2, 32), torch.zeros(3, 2, 32), torch.zeros(3, 4), torch.zeros(3, 8), torch.zeros(3, 32),
            torch.zeros(3, 32)]
    return [
        (outs[:2], lambda **kw: evo.qk_norm_rope(q, k, pos, rope, out=tuple(outs[:2]), **kw)),
        (outs[1:3], lambda **kw: evo.cache_read(cache, tab, one, 3, torch.float32, out=tuple(outs[1:3]), **kw)),
        (outs[:1], lambda **kw: evo.qkv_write(cache, tab, one, q, k, k, rope, q_out=outs[0], **kw)),
        ([outs[0], outs[3]], lambda **kw: evo.chunk_attention(q, cache, tab, one, out=outs[0], lse=outs[3], **kw)),
        ([outs[4]], lambda **kw: evo.linear4(x, w, out=outs[4], **kw)),
        (outs[5:], lambda **kw: evo.block_norm(x, x, x_out=outs[5], h_out=outs[6], **kw))]


@pytest.mark.parametrize("i", range(6))
def test_given_outputs_are_kept_for_the_stream(monkeypatch, i):
    rec = _Record(monkeypatch)
    given, call = _calls()[i]
    call(stream=_Stream(11))
    assert rec.launched and all(h == 11 for _, h in rec.launched)
    for t in given:
        assert (t.data_ptr(), 11) in rec.kept
