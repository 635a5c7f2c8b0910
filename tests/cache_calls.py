"""Calls of attention over the cache that run in blocks of 128 rows: (new, lens, Hq, Hkv, d, page, dtype).  Used by the GPU tests of those blocks and by the host test that
they still run in them."""
import itertools
import random

_SHAPES = [
    # tiles that end anywhere, a last one of a single query, a third sequence shorter than a tile
    ([300, 129, 70], [300, 1000, 90], 32, 16, 64),
    # more queries than keys: rows, and whole tiles, that see nothing
    ([200, 260], [90, 191], 64, 32, 32),
    # long caches in pieces, the second's last pieces behind its end
    ([700, 500], [3000, 1700], 8, 8, 128),
    # three heads to one, a sequence without queries and one without keys, the smallest pages
    ([150, 0, 333, 40], [2000, 50, 2500, 0], 9, 3, 16),
    # the largest pages; one query beside hundreds
    ([129, 1, 400], [5000, 70, 400], 4, 4, 256),
]
LARGE_TILES = [(new, lens, Hq, Hkv, d, page, dtype) for (new, lens, Hq, Hkv, page), d, dtype in itertools.product(_SHAPES, (64, 128), ("bf16", "f32"))]


def any_large(seed):
    """(arguments, causal, layout, rows behind): at least 64 heads of the cache, so that blocks of 128 rows fill the chip on short caches too."""
    r = random.Random(300 + seed)
    n, d = r.choice([1, 2, 3]), r.choice([64, 128])
    Hkv, group = r.choice([64, 70, 128]), r.choice([1, 1, 2, 3])
    new = [r.randint(257, 420) for _ in range(n)]
    lens = [r.choice([1, r.randint(1, 300), r.randint(512, 800)]) for _ in range(n - 1)] + [r.randint(512, 900)]
    call = (new, lens, Hkv * group, Hkv, d, r.choice([16, 32, 64, 128, 256]), r.choice(["bf16", "f32"]))
    return call, r.random() < 0.6, r.choice(["token", "head", "slice"]), r.choice([0, 3])


# (n_seq, total, max_new, Hq, Hkv, d, page, max_pages): tables and lengths of nonsense; pages behind 4 GB
NONSENSE = (3, 700, 700, 64, 64, 64, 16, 40)
BEHIND_4_GB = ([500, 600], [1000, 700], 16, 16, 128, 256, "bf16")
