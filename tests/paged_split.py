"""The split of a paged batch's attention into work items, as csrc/paged.hpp (Plan) makes it,
replayed on the host: which units are cut, and into how many pieces."""
import math

# tile rows: keys of a block, items aimed at, shortest piece in blocks
TILES = {16: (128, 256, 2), 64: (64, 256, 4), 128: (64, 512, 4)}
PART = {16: lambda d: 16 * (d + 2) * 4, 64: lambda d: 64 * (d + 4) * 4, 128: lambda d: 128 * (d + 4) * 4}
SYNC_BYTES = 8192


def tile_rows(new, group, ragged=True):
    mean = sum(new) * group / len(new)
    return 16 if not ragged or mean <= 32 else (64 if mean <= 64 else 128)


def split(lens, new, group, kv_heads, rows, window=0):
    """items, units that are cut, their pieces, the largest number of blocks in a piece."""
    keys, target, least = TILES[rows]
    shares = []
    for n, t in zip(lens, new):
        lo = max(0, min(max(n - t, 0) - (window - 1), n)) if window else 0
        shares.append((-(-t * group // rows) * kv_heads, -(-(n - lo // keys * keys) // keys)))

    def top(b):
        return 128 if rows == 16 else max(1, int(math.sqrt(b) * (2 if rows == 64 else 1)))

    def counts(x):
        p = [(u, min(top(b), max(1, -(-b // x)))) for u, b in shares]
        return sum(u * c for u, c in p), sum(u for u, c in p if c > 1), sum(u * c for u, c in p if c > 1)

    n = sum(u * b for u, b in shares)
    x = max(least, math.ceil(min(n * 1.0001 / target, 1e9)))
    items, units, pieces = counts(x)
    if pieces and target < items <= 4 * target:
        longer = [x, x + x // 4, x + x // 2, 2 * x]
        time = [math.ceil(counts(y)[0] / target) * y for y in longer]
        x = longer[time.index(min(time))]
        items, units, pieces = counts(x)
    return items, units, pieces, x


# Batches (lens, new) whose cut units come to nearly two pieces each of as many units as items are aimed
# at: 5 heads of long sequences just above the longest piece, and so many short ones that the cut stands.
MOST = {16: ([51200] * 50 + [9] * 400, [1] * 450), 64: ([25600] * 50 + [40] * 400, [64] * 50 + [40] * 400),
        128: ([25600] * 101 + [64] * 330, [128] * 101 + [64] * 330)}
MOST_HEADS = 5
