"""Memory that a call on pages may not be given twice: its kernels read some arrays again when they have written others, and by what they read they find their
way in memory.  No GPU: addresses that nothing follows; every call must end before it reaches a launch."""
import pytest

from paper_2203_05016_amd import binding

BAD_SHAPE = -2
HERE = 1 << 20
ROWS, WIDTH, PAGES = 3, 4, 8
CACHE = binding._Cache(128, PAGES, 32, 2, 64, 0)
# where the arrays of one side lie, and how many numbers they hold
ARRAYS = {"table": (0, ROWS * WIDTH), "lengths": (4096, ROWS), "uses": (8192, PAGES)}


def side(at, **kw):
    return binding._Pages(**{**dict(sequences=ROWS, table_pages=WIDTH, table_ld=WIDTH), **{name: at + off for name, (off, _) in ARRAYS.items()}, **kw})


def need():
    return binding.lib().shflbw_kv_pages_workspace(CACHE, ROWS)


def extend(i, o, counts=7 * HERE, slots=6 * HERE, starts=5 * HERE, tokens=9, work=8 * HERE):
    return binding.lib().shflbw_kv_extend(CACHE, i, o, counts, slots, starts, tokens, work, need(), None)


def fork(i, o, parents=7 * HERE, work=8 * HERE):
    return binding.lib().shflbw_kv_fork(CACHE, i, o, parents, work, need(), None)


def compact(i, o, work=8 * HERE):
    return binding.lib().shflbw_kv_compact(CACHE, i, o, work, need(), None)


def ends(base, have, size):
    """Addresses of `size` numbers that share the first or the last of the `have` numbers at base."""
    return base, base + 4 * (have - 1), base - 4 * (size - 1)


@pytest.mark.parametrize("name", ARRAYS)
def test_results_over_what_is_read_again(name):
    """The copies of a fork look up their sources by the parents once lengths, table and uses are written."""
    off, have = ARRAYS[name]
    for at in ends(2 * HERE + off, have, ROWS):
        assert fork(side(HERE), side(2 * HERE), parents=at) == BAD_SHAPE, (name, at)
        assert extend(side(HERE), side(2 * HERE), counts=at) == BAD_SHAPE, (name, at)
        assert extend(side(2 * HERE), side(2 * HERE), counts=at) == BAD_SHAPE, (name, at)


@pytest.mark.parametrize("name", ARRAYS)
def test_slots_and_starts_over_other_arrays(name):
    off, have = ARRAYS[name]
    for base in (HERE, 2 * HERE):
        for kw in ([dict(slots=at) for at in ends(base + off, have, 9)] + [dict(starts=at) for at in ends(base + off, have, ROWS + 1)]):
            assert extend(side(HERE), side(2 * HERE), **kw) == BAD_SHAPE, (name, kw)


def test_slots_and_starts_over_counts_and_each_other():
    for kw in ([dict(slots=at) for at in ends(7 * HERE, ROWS, 9)] + [dict(starts=at) for at in ends(7 * HERE, ROWS, ROWS + 1)] +
               [dict(slots=at) for at in ends(5 * HERE, ROWS + 1, 9)]):
        assert extend(side(HERE), side(2 * HERE), **kw) == BAD_SHAPE, kw


def test_workspace_and_cache_over_arrays():
    """What lies in the workspace is an array's place there: lists of pages, ranks, counts.  The cache's bytes are 128 to 128 + 8 pages of 4352."""
    size = need() // 4
    arrays = [(base + off, have) for base in (HERE, 2 * HERE) for off, have in ARRAYS.values()]
    for at, have in arrays:
        # (multiples of 16, as the workspace has to be)
        for work in (at, at + 4 * (have - 1) & ~15, (at - 4 * (size - 1) + 15) & ~15):
            for call in (extend, fork, compact):
                if call is not compact or at not in (HERE + 4096, 2 * HERE + 4096):          # which has no lengths
                    assert call(side(HERE), side(2 * HERE), work=work) == BAD_SHAPE, (call, hex(at), hex(work))
    for at in (7 * HERE, 6 * HERE, 5 * HERE):
        assert extend(side(HERE), side(2 * HERE), work=at) == BAD_SHAPE
    assert fork(side(HERE), side(2 * HERE), parents=8 * HERE) == BAD_SHAPE
    inside = 128 + 8 * 4352 - 4
    for name in ARRAYS:
        for call in (extend, fork, compact):
            if call is not compact or name != "lengths":
                assert call(side(HERE, **{name: inside}), side(2 * HERE)) == BAD_SHAPE and call(side(HERE), side(2 * HERE, **{name: inside})) == BAD_SHAPE
    assert fork(side(HERE), side(2 * HERE), parents=inside) == BAD_SHAPE and extend(side(HERE), side(2 * HERE), slots=inside) == BAD_SHAPE
    assert compact(side(HERE), side(2 * HERE), work=1024) == BAD_SHAPE
