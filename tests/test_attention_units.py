"""How attention shares out a batch (csrc/attn_units.h), compiled for the host: whatever the lengths are, parts and cut tiles stay
within their lists, and no tile is joined that a workgroup of the grid has not written.  No GPU is needed."""
import ctypes as C
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_17029_amd", "csrc")
SHIM = """
#include "attn_units.h"
using namespace qblora;
extern "C" {
int64_t sum_blocks(int64_t all, int tiles, int blocks) { return add_blocks(all, Cost{tiles, blocks}); }
int64_t per_unit(int64_t all, int target, int least) { return blocks_per_unit(all, target, least); }
void units(int tiles, int blocks, int64_t per, int slack, int* out) {
    const Units u = units_of(Cost{tiles, blocks}, per, slack);
    out[0] = u.tiles; out[1] = u.splits; out[2] = u.count; out[3] = u.cuts;
}
int64_t grid(int64_t tiles, int64_t blocks_of_row, int target, int least) { return units_of_grid(tiles, blocks_of_row, target, least); }
int blocks(int context, int fresh, int limit, int window) { return blocks_of(context_of(context), fresh, limit, window); }
int tile_blocks(int context, int fresh, int limit, int window, int behind) { return blocks_of_tile(context, fresh, limit, window, behind); }
int within(int count, int grid_units) { return units_within(count, grid_units); }
int add(int a, int b) { return add_units(a, b); }
int joined(int cuts, int total, int grid_units) { return cut_tiles(cuts, total, grid_units); }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_units")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    L = C.CDLL(str(d / "shim.so"))
    L.per_unit.argtypes, L.per_unit.restype = [C.c_int64, C.c_int, C.c_int], C.c_int64
    L.units.argtypes = [C.c_int, C.c_int, C.c_int64, C.c_int, C.c_void_p]
    L.grid.argtypes, L.grid.restype = [C.c_int64, C.c_int64, C.c_int, C.c_int], C.c_int64
    return L


# rows of a tile, units aimed at for a key / value head, least blocks of a unit, slack: as launch() has them for 1 to 64 heads
FORMS = [(16, 1024 // kv, 8, 0) for kv in (1, 8, 64)] + [(128, 384 // kv, 16, 1) for kv in (1, 8, 64)]


def share_out(rules, form, starts, T, group, contexts, row_positions):
    """What a call of all requests in one form leaves: units, parts, cut tiles, the cut tiles that are joined, the grid's units."""
    rows, target, least, slack = form
    costs = []
    for i, context in enumerate(contexts):
        s0 = min(max(starts[i], 0), T)
        fresh = min(max(starts[i + 1], s0), T) - s0
        blocks = max(1, -(-min(context + fresh, row_positions) // 32))
        costs.append((-(-fresh * group // rows), blocks) if fresh else (0, 0))
    per = rules.per_unit(sum(t * b for t, b in costs), target, least)
    requests = min(len(contexts), T)
    grid = rules.grid((T * group + requests * (rows - 1)) // rows, row_positions // 32 + 1, target, least)
    out = (C.c_int * 4)()
    total = cuts = units = parts = cut = 0
    for t, b in costs:
        rules.units(t, b, per, slack, out)
        assert out[0] == t and out[1] >= 1 and out[2] == t * out[1]
        if out[1] > 1:
            assert out[1] <= target                                        # the join holds one weight of each part
            parts, cut = parts + out[2], cut + t
        units += out[2]
        total = rules.add(total, rules.within(out[2], grid))
        assert 0 <= total < 1 << 27
        cuts += out[3]
    assert cuts == parts + (cut << 16)
    assert parts <= 2 * target and cut <= target
    return units, parts, cut, rules.joined(cuts, total, grid), grid


def lengths(r, n):
    return [r.choice([0, 1, r.randint(0, 300), r.randint(0, 5000), r.randint(0, 200000)]) for _ in range(n)]


@pytest.mark.parametrize("form", FORMS)
def test_requests_that_follow_each_other_fit_their_grid(rules, form):
    r = random.Random(1)
    some = 0
    for _ in range(1500):
        n, group = r.choice([1, 2, 5, 40, 300]), r.choice([1, 3, 8, 16])
        fresh = [r.choice([0, 1, 1, r.randint(1, 40), r.randint(1, 2000)]) for _ in range(n)]
        starts = [0]
        for m in fresh:
            starts.append(starts[-1] + m)
        contexts = lengths(r, n)
        row = -(-max(c + m for c, m in zip(contexts, fresh)) // 256) * 256 + 256
        units, _, cut, joined, grid = share_out(rules, form, starts, starts[-1], group, contexts, row)
        if starts[-1]:
            assert units <= grid and joined == cut
        some += cut > 0
    assert some > 200


@pytest.mark.parametrize("form", FORMS)
def test_no_tile_is_joined_that_has_not_run(rules, form):
    """Starts in any order count tokens more than once: more units than the grid has, and the tiles of those that never run
    are not in the list."""
    r = random.Random(2)
    more = 0
    for _ in range(1500):
        n, T = r.choice([2, 5, 40, 300]), r.choice([1, 16, 64, 500])
        starts = [r.choice([0, T, r.randint(-5, T + 5), 2**31 - 1]) for _ in range(n + 1)]
        contexts = lengths(r, n)
        units, _, cut, joined, grid = share_out(rules, form, starts, T, r.choice([1, 8]), contexts, r.choice([256, 3072, 300032]))
        assert joined == (cut if units <= grid else 0)
        more += units > grid and cut > 0
    assert more > 20


def test_an_example_of_starts_that_do_not_ascend(rules):
    """Three requests of all 64 tokens, 8 heads each, over 3000 positions: 72 units where the grid has 63."""
    units, _, cut, joined, grid = share_out(rules, (128, 384, 16, 1), [0, 64, 0, 64, 0, 64, 0], 64, 8, [3000] * 6, 3200)
    assert (units, grid, cut, joined) == (72, 63, 12, 0)


@pytest.mark.parametrize("form", FORMS)
def test_units_of_more_blocks_than_32_bits_count(rules, form):
    """Sums of blocks up to 2^60: a tile is at most 2^25 blocks, so a unit of more needs no cut."""
    rows, target, least, slack = form
    out = (C.c_int * 4)()
    sizes = [(1 << k) + d for k in range(20, 61) for d in (-1, 0, 1, 5)] + [target * ((1 << 32) * k + d) for k in (1, 2, 7) for d in (0, 1, 3, 100)]
    for every in sizes:
        per = rules.per_unit(every, target, least)
        for blocks in (1, 100, 4096, 1 << 20, (1 << 25) + 1):
            if blocks > every:
                continue
            rules.units(1, blocks, per, slack, out)
            exact = max(-(-every // target), least)
            assert out[1] == max(1, (blocks + (exact // 2 if slack else exact - 1)) // exact), (every, blocks)
            assert out[1] <= target


def test_batches_of_long_rows_and_many_tokens(rules):
    """2048 requests that all count the same 2048 tokens of 16 heads, over the longest rows there are, in the single tokens' form for 64
    key / value heads: 2^37 blocks in all, 2^33 a unit."""
    for form in FORMS:
        units, parts, cut, _, _ = share_out(rules, form, [0, 2048] * 2049, 2048, 16, [1 << 30] * 4096, 1 << 30)
        assert units >= 4096 // 2 * 2048 * 16 // form[0]


def test_blocks_of_the_longest_requests(rules):
    """Positions behind 2^30 are none of a table: the sums of lengths stay within 32 bits."""
    most = 1 << 30
    for context in (-5, 0, 1, most - 2, most - 1, most, 2 * most - 1):
        for fresh in (1, 33, most - 1, most):
            for limit in (0, 16, 4096, most):
                for window in (0, 1, 4096, most):
                    c = min(max(context, 0), most - 1)
                    hi, lo = min(c + fresh, limit), max(c + 1 - window, 0) if window else 0
                    want = -(-hi // 32) - lo // 32 if hi > lo else 1
                    assert rules.blocks(context, fresh, limit, window) == want, (context, fresh, limit, window)


@pytest.mark.parametrize("rows", [16, 128])
def test_blocks_of_a_tile_are_those_that_it_sees(rules, rows):
    """With a window, a tile of a long request is charged with its own positions: as many blocks as it touches at most, and no more
    than two above what the longest of the request's tiles touches.  It was the whole request's 50 blocks for each tile of
    1500 tokens over 2000 with a window of 64."""
    r = random.Random(3)
    cases = [(2000, 1500, 1 << 20, 64, 3)] + [(r.randint(0, 5000), r.randint(1, 3000), 16 * r.randint(1, 600), r.choice([0, 1, 64, r.randint(1, 6000)]),
                                               r.choice([1, 3, 8, 40, 200])) for _ in range(300)]
    for context, fresh, limit, window, group in cases:
        most = 1
        for row0 in range(0, fresh * group, rows):
            first, last = row0 // group, (min(row0 + rows, fresh * group) - 1) // group
            lo, hi = max(context + first + 1 - window, 0) if window else 0, min(context + last + 1, limit)
            if hi > lo:
                most = max(most, -(-hi // 32) - lo // 32)
        got = rules.tile_blocks(context, fresh, limit, window, (rows - 2 + group) // group)
        assert got >= most, (context, fresh, limit, window, group)
        if window and fresh * group > rows and limit >= context + fresh:
            assert got <= most + 2, (context, fresh, limit, window, group, got, most)
        if not window:
            assert got == rules.blocks(context, fresh, limit, 0)


def test_blocks_of_any_number_of_requests(rules):
    """2^30 requests that all count the most tokens over the longest rows pass 64 bits; a thread adds up 2^22 of them, 256 threads are summed."""
    rules.sum_blocks.argtypes, rules.sum_blocks.restype = [C.c_int64, C.c_int, C.c_int], C.c_int64
    all_ = 0
    for _ in range(5000):
        all_ = rules.sum_blocks(all_, 1 << 27, (1 << 25) + 1)
        assert 0 < all_ * 256 < 1 << 63
    for form in FORMS:
        assert rules.per_unit(all_, form[1], form[2]) == rules.per_unit(1 << 60, form[1], form[2])
    assert rules.sum_blocks(rules.sum_blocks(0, 3, 50), 7, 11) == 3 * 50 + 7 * 11
