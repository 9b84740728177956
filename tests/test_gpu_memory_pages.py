"""GPU parity of chunk attention over parts of a cache that are longer than the
page numbers a wave holds at a time."""
import pytest

from tests.gpu_util import device, say
from tests.memory_util import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt,rows,lengths,heads,dh", [
    ("bf16", "bf16", [40], [4097], 1, 128), ("bf16", "bf16", [40, 33], [9000, 4170], 1, 128), ("bf16", "int8", [100], [8200], 1, 128),
    ("bf16", "bf16", [70], [4200], 1, 64),
    ("bf16", "bf16", [1, 2], [32770, 33500], 1, 64), ("fp32", "fp32", [1], [33000], 1, 32), ("bf16", "fp8", [3], [40000], 1, 64),
    ("fp32", "fp32", [2], [16400], 1, 128)])
def test_pages_of_long_parts(dtype, fmt, rows, lengths, heads, dh):
    """More blocks than the page numbers that a wave holds at a time: 64 for
    itself, of every fourth or eighth block where waves take blocks in turn."""
    say(f"[gpu] pages of long parts {dtype} over {fmt}: rows {rows} lengths {lengths} dh {dh}")
    c = Call(device(), dtype, fmt, rows, lengths, heads, heads, dh, seed=26, causal=True)
    c.check("one part", got=c.run(max_length=1))


def test_pages_of_long_tiles_of_a_wave():
    """The same where a wave has a row tile to itself."""
    lengths = [4200, 64, 8300] + [(37 * s) % 140 for s in range(61)]
    c = Call(device(), "bf16", "int8", [1] * 64, lengths, 16, 16, 32, seed=27)
    c.check("one wave", got=c.run(max_length=1))
