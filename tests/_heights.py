"""The rows of the tile that a call takes (fastest_height in lmhead_tile.h, with the times that the
sources give it): which of them a test's sizes run."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_23866_amd", "csrc")


def _times(name):
    """(alone, each, second) of the one call of fastest_height in a source file."""
    with open(os.path.join(CSRC, name)) as f:
        found = re.findall(r"fastest_height\(\s*\w+,\s*column_tiles\(\w\),\s*\{([^}]*)\},\s*\{([^}]*)\},\s*([\d.]+)\)",
                           f.read())
    (alone, each, second), = found
    return [float(x) for x in alone.split(",")], [float(x) for x in each.split(",")], float(second)


def _height(rows, columns, times):
    alone, each, second = times
    tiles, best, least = -(-columns // 128), 0, 0.0
    for k in range(3):
        bm = 64 << k
        tail = rows % bm
        last = 0 if tail == 0 else 0.75 if k == 2 and tail <= 128 else 1
        per_unit = (rows // bm + last) * tiles / 256
        cost = max(second * alone[k] if per_unit > 1 else alone[k], each[k] * (per_unit + 0.4))
        if best == 0 or cost < least:
            best, least = bm, cost
    return best


def xent(rows, V):
    """Rows of the cross entropy's tile for a block of `rows` rows."""
    return _height(rows, V, _times("xent.hip"))


def mxfp4(M, N):
    """Rows of the four-bit tile (products of more than 32 rows, statistics)."""
    return _height(M, N, _times("mxfp4.hip"))
