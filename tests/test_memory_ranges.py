"""CPU tests of the ranges that chunk attention's arguments have (refused before
any device work)."""
from tests.test_memory_pins import _att, _attend, _cache, _lib, _rows

UNSUPPORTED = -5


def test_refuses_more_rows_than_positions():
    L = _lib()
    one = _cache(n_kv_heads=1)
    for n, code in ((1 << 30, UNSUPPORTED), ((1 << 31) - 2, UNSUPPORTED)):
        assert _attend(L, cache=one, rows=_rows(n_seqs=1, n_rows=n, max_rows=n), att=_att(n_heads=1)) == code
        assert "2^30" in L.evo_last_error().decode()
