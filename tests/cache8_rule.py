"""Which tiles, splits and shares a call of spla_attend8 takes: the library's rule, restated for
tests that have to reach one of them (test_cache8_rule.py holds it to the library's own; not
collected by pytest)."""

from __future__ import annotations

from dataclasses import dataclass

FILL, TILE_FILL, MAX_SPLIT = 512, 768, 128


def ceil_div(a, b):
    return -(-a // b)


@dataclass
class Plan:
    rows: int     # query rows per tile: 16 or 128
    n_tiles: int
    n_split: int  # workgroups that may share a tile's keys
    shares: int   # workgroups that share all sequences' keys by their lengths; 0: none
    join: bool    # whether a launch of its own joins the splits

    @property
    def tiles(self):
        return self.rows == 128


def plan(dtype, batch, hkv, group, cap, T, window=0, sinks=0, prefix=False):
    keys = cap
    if window > 0 and not prefix:
        keys = min(window + sinks + T + 64, cap)
    rows, bh = T * group, batch * hkv
    steps = ceil_div(rows, 16) * bh * ceil_div(keys, 32)
    small = rows <= 64 or steps <= (32768 if dtype == "bf16" else 98304)
    tile = 16 if small else 128
    n_tiles = ceil_div(rows, tile)
    wgs = bh * n_tiles
    n = FILL // wgs if small and FILL // wgs > 1 else TILE_FILL // wgs
    n = max(1, min(n, ceil_div(keys, (4 if small else 16) * 32), MAX_SPLIT))
    joined = 1
    while joined < min(16, rows):
        joined *= 2
    join = n > 1 and (not small or n * joined > 128)
    p = Plan(tile, n_tiles, n, 0, join)
    most = min(512 // joined, MAX_SPLIT)
    if (small and 2 <= batch <= 64 and wgs <= FILL // 4 and keys // 32 >= 64 * n
            and 2 * n <= most):
        p.shares, p.n_split, p.join = FILL, most, False
    return p
