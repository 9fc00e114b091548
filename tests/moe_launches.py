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


# (bits, rows, top_k, experts, hidden, width): between them every instance and every path, most of them short in the other direction
CASES = (
    (1, 1, 2, 4, 512, 4608), (1, 1, 2, 4, 4608, 512), (1, 1, 2, 4, 8704, 512), (1, 3, 1, 2, 512, 8704), (1, 16, 2, 4, 512, 4608),
    (1, 16, 2, 4, 4608, 512), (1, 16, 8, 64, 7680, 512), (1, 16, 8, 128, 512, 7680), (1, 20, 2, 3, 512, 2560), (1, 20, 2, 3, 2560, 512),
    (1, 24, 6, 24, 5120, 512), (1, 70, 8, 40, 512, 4608), (2, 3, 1, 2, 256, 4352), (2, 3, 1, 2, 4352, 256), (2, 5, 2, 4, 256, 8448),
    (2, 12, 8, 64, 7424, 256), (2, 16, 2, 4, 256, 6400), (2, 16, 2, 8, 6400, 256), (2, 16, 4, 32, 2048, 2048), (2, 16, 4, 32, 7424, 256),
    (2, 16, 8, 128, 256, 7424), (2, 16, 8, 128, 512, 2048), (2, 16, 8, 128, 2048, 256), (2, 20, 2, 3, 256, 2560), (2, 20, 2, 3, 2304, 256),
    (2, 70, 8, 40, 512, 4352), (2, 70, 8, 40, 4352, 256), (3, 4, 4, 16, 128, 4224), (3, 4, 4, 16, 4352, 128), (3, 5, 2, 4, 128, 5760),
    (3, 12, 8, 64, 384, 6784), (3, 12, 8, 64, 1408, 1408), (3, 16, 2, 4, 128, 5248), (3, 16, 2, 4, 5248, 128), (3, 16, 4, 32, 5760, 128),
    (3, 16, 8, 64, 1024, 896), (3, 16, 8, 128, 6784, 128), (3, 20, 2, 3, 128, 2176), (3, 40, 4, 16, 2176, 128), (3, 70, 8, 40, 512, 3328),
    (3, 70, 8, 40, 640, 4224), (3, 70, 8, 40, 3328, 256), (4, 3, 1, 2, 128, 7296), (4, 3, 1, 2, 7680, 128), (4, 5, 2, 4, 128, 5760),
    (4, 5, 2, 4, 5760, 128), (4, 16, 2, 4, 128, 5248), (4, 16, 2, 4, 5248, 128), (4, 16, 4, 64, 384, 5760), (4, 16, 8, 128, 5760, 128),
    (4, 20, 2, 3, 1152, 128), (4, 40, 2, 4, 128, 1152), (4, 70, 8, 40, 512, 2048), (4, 70, 8, 40, 640, 1152), (4, 70, 8, 40, 2048, 256),
)
