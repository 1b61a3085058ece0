"""The library holds the tile kernels that a call can reach and no others (nm, no GPU): over pages
only the large row tile is taken, D = 256 has one tile."""
import collections
import re
import subprocess

from paper_2609_04910_amd import attention as at


def test_forward_tiles_in_the_library():
    out = subprocess.run(["nm", "-C", at.LIB_PATH], capture_output=True, text=True, check=True).stdout
    tiles = collections.defaultdict(set)
    for dtype, width, rows, paged in re.findall(r"gs::k_attn_fwd<gs::(\w+), (\d+), (\d+), \d+, (\w+), \w+>", out):
        tiles[dtype, int(width), paged == "true"].add(int(rows))
    for dtype in ("F16", "BF16"):
        for width, rows in ((64, 2), (128, 3), (256, 1)):
            assert tiles.pop((dtype, width, True)) == {rows}
            assert tiles.pop((dtype, width, False)) == {rows, max(rows - 1, 1)}
    assert not tiles
