"""Which instance of the experts' row kernel a call takes, by the rules at `launch_product` and `launch_few` in csrc/kmq_moe.hip written out again, and
which of its paths the call goes through.  For tests that say which of them they are for."""
from collections import namedtuple

UNIT = {1: 512, 2: 256, 3: 128, 4: 128}                # columns of a super-block
MOST_ROWS = 128

# as the kernel's template arguments; `gated`: gate and up, else down
Instance = namedtuple("Instance", "bits tokens rows waves teams gated")


def _few(bits, tokens, pairs, experts, columns, blocks, gated):
    units, items = columns // UNIT[bits], min(pairs, experts) * blocks
    if tokens == 4 and items <= 512 and units >= 16:
        waves, all_waves = 8, 8
    elif bits == 4:
        waves, all_waves = 4, 8
    elif units < 16 and items >= 2048:
        waves, all_waves = 2, 4
    else:
        waves, all_waves = 4, 4
    return Instance(bits, tokens, 16, waves, all_waves // waves, gated)


def instance(bits, rows, top_k, experts, hidden, width, gated):
    pairs = rows * top_k
    columns, blocks = (hidden, width // 16) if gated else (width, hidden // 32)
    if rows <= 4 or (rows <= 16 and 2 * pairs <= (6 if bits == 1 else 3) * experts):
        return _few(bits, 4, pairs, experts, columns, blocks, gated)
    if bits > 1 and (rows <= 8 or (rows <= 16 and pairs <= 3 * experts)):
        return _few(bits, 8, pairs, experts, columns, blocks, gated)
    if rows <= 16:
        return Instance(bits, 16, 16, 2, 2, gated)
    all_waves = 8 if bits == 1 else 16
    items = (min(pairs, experts) + pairs // 16) * (width // 128 if gated else hidden // 256)
    waves = 8 if items <= 128 else all_waves // (8 if gated or hidden % 256 == 0 else 4)
    return Instance(bits, 16, MOST_ROWS, waves, all_waves // waves, gated)


def piece(i):
    """Columns whose scales, and tokens above 16 rows, are in shared memory at a time."""
    return 4096 if i.rows <= 16 else 1024 if i.bits == 4 else 2048


def ahead(i):
    """Super-blocks that a wave has asked for before it multiplies."""
    steps = UNIT[i.bits] // 32
    staged = i.rows > 16
    words = 2 * steps * i.bits // 4 + (0 if staged or (i.bits == 1 and i.tokens == 16) else i.tokens // 4 * steps)
    return 2 if staged or words > 10 else 3


def paths(i, columns):
    """What rows of that many columns make an instance go through: the steady loop (a wave that has twice as many super-blocks of a piece as it asks for
    ahead), a second piece, the steady loop in a piece that is not the first."""
    size, unit, out = piece(i), UNIT[i.bits], set()
    for first in range(0, columns, size):
        some = min(size, columns - first) // unit
        most = max(some * (m + 1) // i.waves - some * m // i.waves for m in range(i.waves))
        if first:
            out.add("piece")
        if most >= 2 * ahead(i):
            out.add("loop again" if first else "loop")
    return out


def both(bits, rows, top_k, experts, hidden, width):
    """The two launches of a call: (instance, its paths)."""
    for gated in (True, False):
        i = instance(bits, rows, top_k, experts, hidden, width, gated)
        yield i, paths(i, hidden if gated else width)


def reachable():
    """Every instance that a call can take, with all paths that calls can make it go through."""
    found = {}
    for bits, unit in UNIT.items():
        sizes = [unit * n for n in sorted({*range(1, 20), 8 * 512 // unit, 8 * 512 // unit + 1, 16 * 512 // unit, 16 * 512 // unit - 1, 65536 // unit})]
        for rows in (1, 3, 4, 5, 8, 9, 16, 17, 128):
            for top_k, experts in ((1, 1), (1, 4), (2, 3), (2, 8), (8, 8), (8, 16), (16, 24), (8, 64), (8, 128), (16, 1024)):
                for hidden in sizes:
                    for width in sizes:
                        for i, how in both(bits, rows, top_k, experts, hidden, width):
                            found.setdefault(i, set()).update(how)
    return found
