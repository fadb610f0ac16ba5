"""Which way a gradient of a lookup takes, by the sizes of the call: the rule of the library written down once more, so that tests can
say which form they reach.  `bytes` is the workspace that such a call asks for; test_embed_plan.py holds it against the library's own."""
from dataclasses import dataclass


def _up(x, step):
    return (x + step - 1) // step * step


@dataclass
class Plan:
    form: str                       # "few", "table", "once" (ids grouped by one launch) or "sort" (a stable radix sort)
    by_row: bool = False            # few, not added: a workgroup for each row (otherwise for each id)
    lanes: int = 0                  # of a team that sums rows
    vectors: int = 1                # of four columns, for each lane
    passes: int = 0                 # of the sort
    tile: int = 0
    scanned: bool = False           # the sort's counts are added up by a launch of their own
    rows: int = 0                   # of a grouping workgroup
    chunk: int = 0                  # ids that a team sums
    per_wave: int = 0               # chunks of a joining wave
    bytes: int = 0


def plan(n: int, N: int, d: int) -> Plan:
    lanes = 16 if d <= 64 else 32 if d <= 128 else 64
    if n <= 3500 or (n <= 8192 and N <= n // 4):
        return Plan("few", by_row=n > 0 and (N < n or N <= 4096), lanes=lanes)
    dp, teams = _up(d, 4), 256 // lanes
    lds = (min(N, 65535) + 1) * (teams * dp + 1) * 4
    if 4 <= d <= 256 and lds <= (156 if lanes <= 32 else 80) * 1024:
        blocks = min(256 if lds > 80 * 1024 else 512, -(-n // (16 * teams)))
        return Plan("table", lanes=lanes, bytes=_up(blocks * N * dp * 4, 256) + _up(blocks * N * 4, 256))
    bits, most = N.bit_length(), 9 if n <= 131072 else 11
    passes = max(1, -(-bits // most))
    bits = max(1, -(-bits // passes))
    tile = 512 if n <= 65536 else 1024 if n <= 262144 else 4096
    tiles = -(-n // tile)
    chunk = 8
    while chunk < 256 and n // chunk > 4096:
        chunk *= 2
    chunks = -(-n // chunk)
    rows = -(-N // 256)
    once = n <= (16384 if passes == 1 else 49152) and rows <= 1024 and 64 * rows + 32 * (-(-n // 1024) * 64) <= 156 * 1024
    pairs = [n * 8, n * 4] if once else [n * 8] * min(passes, 2) + [(tiles << bits) * 4, 4 << bits]
    parts = pairs + [chunks * dp * 4] * 2
    return Plan("once" if once else "sort", lanes=lanes, vectors=1 if d <= 256 else 2 if d <= 512 else 4, passes=passes, tile=tile,
                scanned=(tiles << bits) > (16384 if n <= 262144 else 4096), rows=rows, chunk=chunk, per_wave=min(64, -(-chunks // 16384)),
                bytes=sum(_up(p, 256) for p in parts))
