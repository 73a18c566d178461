"""Reads of the per-token arrays in the norm + rotation kernels stay inside them.

A launch rounds its warps up to whole blocks, so a warp's first token may lie past the last one:
every read of `slots` and `pos` has to be behind a comparison of its own index with the number of
tokens.  The arrays' owners need not align or pad them, and a value read past the end is not used,
so no output shows such a read: the source is checked instead."""
import os
import re

from paper_2609_13141_gb300 import _build

SOURCE = os.path.join(_build.CSRC, "k_rope.cu")


def _warps_without_a_token(T, heads, rows_per_warp, warps=8):
    """Launch geometry of few tokens: the start tokens of a launch's warps that are past the last token."""
    parts = -(-heads // rows_per_warp)
    total = -(-T * parts // warps) * warps
    step = total // min(parts, total)
    starts = [w // min(parts, total) for w in range(total)]
    return [t for t in starts if T <= t < step]


def test_some_warps_start_past_the_last_token():
    # why the guard is needed: 8 + 2 x 1 heads of 64 (16 rows a warp), one token; 8 + 2 x 2 of 128 (8 rows), one
    assert _warps_without_a_token(1, 10, 16) == list(range(1, 8))
    assert max(_warps_without_a_token(1, 12, 8)) == 3


def test_every_read_of_a_per_token_array_is_behind_its_bound():
    src = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    reads = list(re.finditer(r"load\(a\.(?:slots|pos) \+ ([^()]+)\)", src))
    assert len(reads) >= 4
    for m in reads:
        index = re.escape(m.group(1).strip())
        # the statement itself, or a return ahead of it in the same block
        before = src[max(0, m.start() - 200):m.start()]
        guard = rf"{index} < a\.T\)?[^;{{}}]*$|if \({index} >= a\.T\) return;[^{{}}]*$|if \({index} < a\.T\) \{{[^{{}}]*$"
        assert re.search(guard, before), f"unguarded: {before[-60:]}{m.group(0)}"
