"""The helper that says what a CTA of the attention's tile kernel has to do: its constants are the kernel's, and nothing is left out or done twice."""
import os
import random
import re

from tests import kv_line

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_05528_b200", "csrc")


def test_constants():
    tile, cache = (open(os.path.join(CSRC, f)).read() for f in ("kv_attend_tcgen05.cu", "kv_cache.cuh"))
    assert int(re.search(r"HALF = (\d+), ROWS = 2 \* HALF", tile).group(1)) * 2 == kv_line.ROWS
    assert int(re.search(r"KEYS = (\d+)", tile).group(1)) == kv_line.KEYS
    assert int(re.search(r"OVERHEAD = (\d+)", tile).group(1)) == kv_line.OVERHEAD
    assert int(re.search(r"SEQS = (\d+)", tile).group(1)) == kv_line.SEQS
    assert int(re.search(r"KV_FEW_ROWS = (\d+)", cache).group(1)) == kv_line.FEW_ROWS


def test_shares():
    rng = random.Random(1)
    for _ in range(100):
        sizes = []
        for _ in range(rng.randint(1, 40)):
            length = rng.randint(1, 900)
            sizes.append((rng.randint(0, length), length))
        heads, group, window = rng.choice((1, 2, 8)), rng.choice((1, 4, 5)), rng.choice((0, 0, 100))
        rows = [n * group for n, _ in sizes if n * group > kv_line.FEW_ROWS]
        if not rows:
            continue
        cut, uncut = (kv_line.shares(sizes, heads, group, window=window, whole=w) for w in (False, True))
        assert sum(map(len, uncut)) == heads * sum(-(-r // kv_line.ROWS) for r in rows)
        assert sum(b for s in cut for b, _ in s) == sum(b for s in uncut for b, _ in s)
    assert kv_line.shares([(64, 64)], 1, 1) == [[(1, 1)]] + [[]] * 5
    # a unit of 148 blocks and its overhead: 153 steps, 76 and 77, of which the second has the overhead
    assert kv_line.shares([(256, 64 * 148)], 1, 1, n_ctas=2) == [[(76, 2)], [(72, 2)]]
