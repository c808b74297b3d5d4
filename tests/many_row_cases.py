"""Calls of delta_extend_attn that its plan sends to the kernel of 256-row tiles (a host test holds that they
still go there): (tokens held, new tokens, query heads, KV heads), for both head sizes and cache types."""
MANY_ROWS = [
    # a long run beside single tokens: tiles of 256 rows that single tokens' rows straddle (5 heads a
    # group), tiles of at most 32 rows (the singles, and the run's last), three pieces of the keys
    ((1300, 400, 30, 900), (1200, 1, 1, 1), 10, 2),
    ((1500, 33, 700), (1500, 1, 0), 14, 2),
    ((1600, 64), (1600, 2), 16, 2),
    ((2300, 50, 2000), (2300, 1, 1), 6, 2),
    # one query head a group, two sequences in two pieces
    ((2600, 2600), (2600, 2600), 4, 4),
    # several sequences, one piece
    ((900, 850, 700, 901), (900, 850, 700, 640), 32, 8),
    # a run longer than its sequence: its first 400 rows see nothing
    ((1000, 50), (1400, 3), 16, 2),
    # 6150 rows: the run's last tile has 6
    ((1230,), (1230,), 10, 2),
    # a chunk behind a long prefix, beside a run of one whole tile less its last row
    ((5000, 100), (600, 63), 16, 4),
    ((3000, 3000, 3000), (700, 1, 700), 16, 2),
    ((1200, 900, 800), (1200, 900, 800), 8, 1),
    ((3000,), (3000,), 4, 2),
]

# ... of one sequence, for values of tokens that a row does not see: a prefix of 200 tokens, three pieces
HIDDEN = ((1500, 20), (1300, 3), 10, 2)

# ... of very many short runs, which would be too many tiles of 32 rows: sequences, tokens held (up to), new
MOST_TILES = (16384, 24, 16, 8, 1)


def plan_call(lens, new, hq, hkv, d):
    """The arguments that the plan goes by: batch, heads, head size, bound, rows, longest run."""
    return len(lens), hq, hkv, d, max(lens), sum(new), max(new)
