"""Calls of attention behind shared prefixes, one for each way that the kernels share the work, and which way that is: the plan is held to it without a GPU, the
results to the definition with one."""

FIELDS = "decode col_tiles waves col_blocks splits split_tiles groups tiny".split()


class Case:
    """families: sequences of every prefix, whose lengths are `prefix`; counts: queries of each sequence; most: what the host says is the longest
    prefix (the table has room for it), where that is not the longest there is."""

    def __init__(self, name, q_heads, heads, D, fmt, families, prefix, own, counts, plan, most=None, page=32):
        self.name, self.q_heads, self.heads, self.D, self.fmt, self.page = name, q_heads, heads, D, fmt, page
        self.families, self.prefix, self.own, self.counts = families, prefix, own, counts
        self.most, self.plan = most or max(prefix), plan

    @property
    def sharing(self):
        """Columns of q that any prefix's sequences have together."""
        starts = [sum(self.families[:g]) for g in range(len(self.families) + 1)]
        return max(sum(self.counts[a:b]) for a, b in zip(starts, starts[1:]))

    def host(self):
        """What the host knows of the call."""
        return dict(prefixes=len(self.families), max_sharing=self.sharing, max_prefix=self.most, batch=len(self.own), heads=self.heads, group=self.q_heads // self.heads,
                    D=self.D, tokens=sum(self.counts), max_queries=max(self.counts), max_length=max(self.own), keys_fit=1)


def _spread(n, low, high):
    """n numbers between low and high, in no order, both ends among them."""
    return [high if i == 1 else low + 7 * i % (high - low + 1) for i in range(n)]


def tiles(waves=8, **kw):
    return dict(decode=0, waves=waves, **kw)


def columns(n, waves=None, **kw):
    return dict(decode=1, col_tiles=n // 16, **({} if waves is None else dict(waves=waves)), **kw)


CASES = [
    # prefixes in blocks of 48 columns, the GPU full of them: 8 x 3 queries of groups of 4, two blocks; groups of 5, of which a block takes 9 queries
    Case("blocks of 48", 4, 1, 96, "f16", [8] * 86, _spread(86, 1, 70), _spread(688, 1, 9), [3] * 688, most=3000,
         plan=dict(behind=0, joins=1, prefix=columns(48, col_blocks=2), own=columns(16, 4))),
    Case("blocks of 48 that a group does not divide", 5, 1, 64, "bf16", [9] * 130, _spread(130, 1, 40), _spread(1170, 1, 5), [1] * 1170, most=2000,
         plan=dict(behind=0, joins=1, prefix=columns(48, col_blocks=1), own=columns(16, 4))),
    # single tokens of so many sequences and heads that workgroups of 4 wavefronts attend to own keys and join
    Case("joined by 4 wavefronts", 8, 8, 64, "f16", [65], [70], _spread(65, 1, 20), [1] * 65, most=2100,
         plan=dict(behind=0, joins=1, prefix=columns(32), own=columns(16, 4))),
    Case("joined by 4 wavefronts, heads of 128", 32, 16, 128, "bf16", [20, 0, 15], [70, 9, 33], _spread(35, 1, 12), [1] * 35, most=1000,
         plan=dict(behind=0, joins=1, prefix=columns(32), own=columns(16, 4))),
    # two, three and four tiles of 16 columns whose last is not full, and blocks of 32, joined with the prefixes' parts
    Case("two tiles joined", 32, 8, 64, "f16", [3, 2, 2, 1], [300, 40, 65, 1], _spread(8, 1, 60), [5, 1, 3, 5, 5, 2, 0, 5], most=17000,
         plan=dict(behind=0, joins=1, prefix=columns(32), own=columns(32))),
    Case("three tiles joined", 40, 8, 64, "bf16", [3, 2, 2, 1], [300, 40, 65, 1], _spread(8, 1, 60), [9, 1, 3, 7, 9, 2, 0, 9], most=17000,
         plan=dict(behind=0, joins=1, own=columns(48))),
    Case("three tiles joined, heads of 96", 40, 8, 96, "f16", [3, 2, 2, 1], [70, 40, 65, 1], _spread(8, 1, 60), [9, 1, 3, 7, 8, 2, 0, 9], most=17000,
         plan=dict(behind=0, joins=1, own=columns(48))),
    Case("four tiles joined", 100, 2, 64, "f16", [10, 10], [100, 33], _spread(20, 1, 60), [1] * 20, most=27000,
         plan=dict(behind=0, joins=1, prefix=tiles(), own=columns(64))),
    Case("blocks of 32 joined", 56, 8, 128, "bf16", [3, 2, 2, 1], [100, 40, 65, 1], _spread(8, 1, 60), [8, 1, 3, 7, 8, 2, 0, 8], most=8500,
         plan=dict(behind=0, joins=1, own=columns(32, col_blocks=2))),
    Case("three blocks of 32 joined", 64, 8, 96, "f16", [3, 2, 2, 1], [100, 40, 65, 1], _spread(8, 1, 60), [9, 1, 3, 7, 8, 2, 0, 9],
         plan=dict(behind=0, joins=1, own=columns(32, col_blocks=3))),
    # own keys by the tile kernel after a launch over prefixes, in one part and in several, by 8 wavefronts and by 4
    Case("tiles, one part", 32, 2, 64, "f16", [2, 1], [90, 33], [70, 9, 150], [9, 10, 17], plan=dict(behind=0, joins=0, own=tiles(splits=1))),
    Case("tiles, several parts", 32, 2, 128, "bf16", [2, 1], [200, 33], [700, 9, 900], [9, 10, 17], plan=dict(behind=0, joins=0, own=tiles())),
    Case("tiles, heads of 96", 18, 1, 96, "f16", [1, 1, 1], [64, 0, 31], [5, 700, 64], [9, 19, 12], plan=dict(behind=0, joins=0, own=tiles())),
    # a part of a prompt among single tokens: the prefix once for all columns, if it is long; prompts and shorter ones, which are much alike
    Case("one of 70 among single tokens", 8, 2, 64, "f16", [12], [150], _spread(12, 1, 90), [1] * 5 + [70] + [1] * 6, most=4000,
         plan=dict(behind=0, joins=0, prefix=tiles(), own=tiles())),
    Case("one of 70 among single tokens, of three prefixes", 10, 2, 128, "bf16", [4, 0, 8], [70, 9, 100], _spread(12, 1, 90), [1, 0, 1, 70] + [1] * 6 + [0, 3], most=3000,
         plan=dict(behind=0, prefix=tiles())),
    Case("one of 70 among single tokens behind a short prefix", 8, 2, 64, "bf16", [12], [150], _spread(12, 1, 90), [1] * 5 + [70] + [1] * 6,
         plan=dict(behind=1, own=tiles())),
    Case("prompts of 20 to 40", 4, 2, 96, "f16", [2, 3], [150, 90], _spread(5, 1, 90), [20, 40, 33, 30, 31], most=2000, plan=dict(behind=1, own=tiles(4))),
]
