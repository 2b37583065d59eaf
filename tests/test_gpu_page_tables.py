"""Block tables, slots and positions made on the GPU against the same request by request on the host: whole numbers, equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _check(context, fresh, page, width, tokens, n_free=None, seed=0):
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    r = np.random.Generator(np.random.Philox(key=[seed, 21]))
    n = len(context)
    held = [min(-(-max(c, 0) // page), width) for c in context]
    wanted = sum(max(0, min(-(-(max(c, 0) + max(m, 0)) // page), width) - -(-max(c, 0) // page)) for c, m in zip(context, fresh))
    n_free = wanted + 5 if n_free is None else n_free
    ids = r.permutation(sum(held) + n_free).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = ids[at:at + h]
        at += h
    free = ids[at:at + n_free]
    want = du.tables(context, fresh, page, free, table, tokens)
    print(f"tables n={n} page={page} width={width} tokens={tokens} free={n_free}", flush=True)
    t = du.dev_i32(table)
    starts, positions, slots, taken = qb.qblora_page_tables(du.dev_i32(context), du.dev_i32(fresh), page, du.dev_i32(free), t, tokens)
    torch.cuda.synchronize()
    for name, got, ref in zip(("table", "starts", "positions", "slots"), (t, starts, positions, slots), want):
        assert np.array_equal(got.cpu().numpy(), ref), name
    assert int(taken) == want[4]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_ragged_batches(page):
    r = np.random.Generator(np.random.Philox(key=[page, 1]))
    for n in (1, 2, 37, 300):
        context = r.integers(0, 700, n)
        fresh = np.where(r.random(n) < 0.5, 1, r.integers(0, 200, n))
        total = int(fresh.sum())
        _check(context, fresh, page, 1024 // page + 2, total, seed=n)
        _check(context, fresh, page, 1024 // page + 2, total + 13, seed=n)


def test_page_boundaries():
    """Contexts and new tokens that end on, before and behind a page; requests with nothing new, with nothing at all."""
    ctx = [0, 0, 15, 15, 16, 16, 17, 31, 32, 0, 48]
    new = [0, 1, 1, 2, 0, 1, 15, 1, 16, 33, 0]
    _check(ctx, new, 16, 4, sum(new))
    _check(ctx[::-1], new[::-1], 16, 4, sum(new) + 1)


def test_more_requests_than_groups_in_lds():
    """Searches that end in a walk through a group's lengths."""
    r = np.random.Generator(np.random.Philox(key=[5, 1]))
    for n in (2047, 2048, 2049, 5000, 12289):
        context, fresh = r.integers(0, 60, n), r.integers(0, 4, n)
        _check(context, fresh, 16, 5, int(fresh.sum()) + 3, seed=n)


def test_free_list_used_up_and_rows_too_short():
    ctx, new = [10, 100, 0, 30], [50, 1, 40, 200]
    for n_free in (0, 1, 4, 9):
        _check(ctx, new, 16, 32, sum(new), n_free=n_free)
    _check(ctx, new, 16, 7, sum(new))                    # the last request's row ends: no pages, no slots behind it
    _check([200], [5], 16, 7, 5)                         # already behind its row
    _check([112], [5], 16, 7, 5)


def test_less_room_than_tokens():
    _check([5, 9, 40], [20, 30, 10], 16, 8, 25)
    _check([5, 9, 40], [20, 30, 10], 16, 8, 0)


def test_lengths_below_zero_count_as_zero():
    _check([-5, 9, -1], [3, -30, 10], 16, 8, 20)


def test_no_requests():
    _check([], [], 16, 3, 9)


def test_largest_lengths():
    """Sums that pass 32 bits keep to their arrays."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    big = 2**31 - 1
    t = du.dev_i32(np.full((3, 2), -1))
    starts, positions, slots, taken = qb.qblora_page_tables(du.dev_i32([big, 0, 3]), du.dev_i32([big, big, 7]), 16,
                                                            du.dev_i32(np.arange(4)), t, 100)
    torch.cuda.synchronize()
    assert starts.tolist() == [0, 100, 100, 100] and (slots.cpu() == -1).all()
    assert positions.tolist() == [big] * 100            # held at the largest number
    assert t.tolist() == [[-1, -1], [0, 1], [-1, -1]] and int(taken) == 2


def test_replays_of_a_graph_and_another_stream():
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    ctx, new, page = np.array([3, 40, 0]), np.array([20, 1, 17]), 16
    table = np.array([[7, -1, -1, -1], [1, 2, 3, -1], [-1] * 4], np.int32)
    free = np.array([9, 8, 6, 5], np.int32)
    context, fresh, frees, t = du.dev_i32(ctx), du.dev_i32(new), du.dev_i32(free), du.dev_i32(table)
    outs = qb.qblora_page_tables(context, fresh, page, frees, t, 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            qb.qblora_page_tables(context, fresh, page, frees, t, 64, *outs)
    for k in range(3):
        new2 = new + k
        fresh.copy_(torch.from_numpy(new2.astype(np.int32)))
        t.copy_(torch.from_numpy(table))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = du.tables(ctx, new2, page, free, table, 64)
        for got, ref in zip((t, *outs), want):
            assert np.array_equal(got.cpu().numpy().reshape(-1), np.asarray(ref).reshape(-1))
