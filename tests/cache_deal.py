"""How attention over the cache deals a call out: the host's part, from its shapes (the workspace's
size follows from it), and the device's, from the lengths."""
from dataclasses import dataclass


def up(a, b):
    return -(-a // b)


@dataclass
class Deal:
    many: bool        # rows rebuilt tiles are shared by
    half: bool        # up to eight rows
    waves: int
    rows: int         # of a row tile
    units: int        # row tiles of all sequences
    merge: bool       # sequences are split
    target: int       # most chunks
    least: int        # blocks of a chunk at least
    items: int        # workgroups
    workspace: int


def deal(B, Hq, H, n, D, cols, page, window=1 << 30, sinks=0):
    r = n * (Hq // H)
    half, many = r <= 8, r > 32
    waves = (8 if r > 128 else 4) if many else 8 if half and B * H <= 128 else 4
    rows = 32 * waves if many else 8 if half else 16 if r <= 16 else 32
    units = B * up(r, rows)
    held = cols * page // 32
    seen = min(held, up(min(window, held * 32) + min(n, rows), 32) + 1
               + up(min(sinks, held * 32), 32))
    least = 16 if many else 32
    merge = seen > least and units <= 256
    items, target, space = units * H, 0, 0
    if merge:
        slots = 256 if waves == 8 or (rows == 32 and D == 128 and not many) else 512
        rounds = max(1, up(2 * items, slots))
        if many and items * seen >= 64 * 2 * slots:
            rounds = max(2, rounds)
        target = slots * rounds
        items = min(target, items * up(seen, least))
        space = items * rows * (D + 2) * 4 + units * 8
    return Deal(many, half, waves, rows, units, merge, target, least, items, space)


def blocks_seen(d, lens, n, group, cols, page, window=1 << 30, sinks=0):
    """Blocks of 32 tokens that each row tile sees."""
    held, out = cols * page // 32, []
    for L in lens:
        for row0 in range(0, up(n * group, d.rows) * d.rows, d.rows):
            lo = L - n + row0 // group
            hi = L - n + (min(row0 + d.rows, n * group) - 1) // group
            near = max(0, lo - window + 1)
            first = min(near // 32, up(min(sinks, near), 32), held)
            out.append(0 if hi < 0 else first + max(0, min(hi // 32 + 1, held) - near // 32))
    return out


def chunks(d, H, seen):
    """The blocks of a chunk, whether that is the second size tried, and each row tile's chunks."""
    blocks = sum(up(t, 8) for t in seen) * 8 * H
    size = lambda parts: up(max(up(blocks, parts), d.least), 8) * 8
    count = lambda c: [max(1, up(t, c)) for t in seen]
    c = size(d.target)
    second = sum(count(c)) * H > d.target
    if second:
        c = size(d.target - d.units * H)
    return c, second, count(c)
