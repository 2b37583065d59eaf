"""Attention over the paged cache against 64-bit softmax, row by row.

An output before it is stored: the weights are rounded to bf16 (8 significant bits: 2^-8 of each at most), the scores are fp32
sums of 64 to 256 products of bf16 values (2e-5 of a weight at the sizes here), so it is off by at most 2^-8 + 2e-5 of the
weighted sum of |v|.  lse: 1e-4."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0**-8 + 2e-5


def _run(b, scale, window=0, max_new=None, **kw):
    from paper_2407_17029_amd import binding as qb
    a = b.device()
    T, heads = a["q"].shape[:2]
    lse = torch.full((T, heads), 5.0, dtype=torch.float32, device=a["q"].device)
    out = torch.full(tuple(a["q"].shape), 9.0, dtype=torch.bfloat16, device=a["q"].device)
    print(f"attention T={T} heads={heads}/{b.k.shape[2]} dim={b.k.shape[3]} page={b.page} contexts={list(b.context)[:6]} "
          f"fresh={list(b.fresh)[:6]} window={window}", flush=True)
    qb.qblora_paged_attention(**a, scale=scale, window=window, max_new=max_new, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


def _check(b, window=0, scale=None, max_new=None):
    import decoder_util as du
    scale = b.q.shape[2] ** -0.5 if scale is None else scale
    out, lse = _run(b, scale, window, max_new)
    want, want_lse, mag = b.expected(scale, window)
    du.assert_bf16(out, want, WEIGHTS * mag, "out")
    got = lse.cpu().numpy().astype(np.float64)
    fine = np.isfinite(want_lse)
    assert np.array_equal(got[~fine], want_lse[~fine], equal_nan=True)
    assert (np.abs(got[fine] - want_lse[fine]) <= 1e-4).all()
    return out


def _batch(*a, **k):
    import decoder_util as du
    return du.Batch(*a, **k)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (8, 1, 64), (6, 2, 128), (4, 2, 256), (3, 3, 64), (40, 2, 64)])
def test_single_tokens(heads, kv_heads, dim, page):
    """Contexts of all lengths around steps and pages, one token each."""
    ctx = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 300, 511, 700]
    _check(_batch(page + heads, ctx, [1] * len(ctx), page, heads, kv_heads, dim), max_new=1)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 128), (8, 2, 128), (4, 1, 64), (2, 1, 256), (20, 1, 64)])
@pytest.mark.parametrize("ctx,new", [([0], [1]), ([0], [70]), ([5, 40, 0], [3, 1, 130]), ([100, 16], [33, 32]), ([257, 0, 64], [65, 2, 64])])
def test_chunks(ctx, new, heads, kv_heads, dim, page):
    _check(_batch(sum(new) + heads, ctx, new, page, heads, kv_heads, dim))


@pytest.mark.parametrize("ctx,new", [([3000, 0, 20, 5000, 7], [1, 1, 1, 1, 1]), ([2500, 9], [40, 3]), ([6000], [1])])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 1)])
def test_long_contexts_are_joined(ctx, new, heads, kv_heads):
    """Long next to short: parts in the workspace, summed by the second launch."""
    _check(_batch(17, ctx, new, 16, heads, kv_heads, 128))


@pytest.mark.parametrize("window", [1, 2, 17, 64, 100, 5000])
@pytest.mark.parametrize("ctx,new", [([0, 300, 90, 64], [1, 1, 1, 1]), ([200, 0, 1500], [150, 60, 2])])
def test_windows(window, ctx, new):
    _check(_batch(window, ctx, new, 32, 4, 2, 128), window=window)


def test_a_wrong_max_new_costs_no_result():
    b = _batch(3, [50, 900, 0], [90, 1, 20], 16, 8, 2, 128)
    for max_new in (0, 1, 5, 90, 100000):
        _check(b, max_new=max_new)


def test_requests_without_new_tokens_and_none_at_all():
    from paper_2407_17029_amd import binding as qb
    _check(_batch(4, [50, 0, 7, 0, 90], [0, 0, 3, 1, 0], 16, 4, 4, 64))
    b = _batch(4, [50, 9], [0, 0], 16, 4, 4, 64)
    a = b.device()
    assert qb.qblora_paged_attention(**a, scale=1.0).shape == (0, 4, 64)
    a["table"], a["starts"], a["context"] = a["table"][:0], a["starts"][:1], a["context"][:0]
    qb.qblora_paged_attention(**a, scale=1.0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [300, 1025])
def test_many_requests(n):
    """More requests than a workgroup has threads."""
    r = np.random.Generator(np.random.Philox(key=[n, 2]))
    _check(_batch(n, list(r.integers(0, 60, n)), [1 if x < 0.9 else 5 for x in r.random(n)], 16, 2, 1, 64))


def test_pages_that_the_table_does_not_list():
    """Holes, numbers outside the cache, and rows that are too short hide their positions; a row that sees nothing is 0."""
    b = _batch(5, [200, 90, 10, 600], [1, 40, 2, 1], 16, 4, 2, 128, width=30)
    b.table[0, 3], b.table[0, 7] = -1, 10**6
    b.table[1, 0], b.table[1, 5] = -7, len(b.k)
    b.table[2, :] = -1
    _check(b)
    _check(b, window=24)
    b.table[0, 1:] = -1                                             # nothing within the window
    _check(b, window=50)


def test_padding_rows_are_left():
    from paper_2407_17029_amd import binding as qb
    import decoder_util as du
    b = _batch(6, [30, 40], [3, 2], 16, 2, 2, 64)
    a = b.device()
    a["q"] = torch.cat([a["q"], torch.full((4, 2, 64), float("nan"), dtype=torch.bfloat16, device=du.DEV)])
    out = torch.full((9, 2, 64), 9.0, dtype=torch.bfloat16, device=du.DEV)
    qb.qblora_paged_attention(**a, scale=0.125, out=out)
    torch.cuda.synchronize()
    assert (out[5:] == 9.0).all() and (out[:5] != 9.0).any()


@pytest.mark.parametrize("heads,kv_heads,ctx,new", [(4, 4, [70, 20], [1, 1]), (8, 2, [40, 0, 333], [60, 20, 3]), (2, 1, [500], [150])])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_unseen_values_do_not_matter_and_seen_ones_do(heads, kv_heads, ctx, new, bad):
    """NaN or an infinity in the key or the value of one position: rows that see it have what the formula gives, those in
    front of it and other heads are as without it."""
    import decoder_util as du
    for which in "kv":
        b = _batch(8, ctx, new, 16, heads, kv_heads, 64)
        i = int(np.argmax(b.fresh))
        p = int(b.context[i] + b.fresh[i] // 2)
        arr = b.k if which == "k" else b.v
        arr[b.table[i, p // 16], p % 16, 0, 3] = bad
        if which == "v":
            arr[b.table[i, p // 16], p % 16, 0, 40] = -bad
        out, _ = _run(b, 0.125)
        want, _, mag = b.expected(0.125)
        got = du.host(out)
        row = int(b.starts[i] + b.fresh[i] // 2)
        sees = np.zeros(b.T, bool)
        sees[row:b.starts[i + 1]] = True
        g = heads // kv_heads
        clean = ~sees
        du.assert_bf16(got[clean], want[clean], WEIGHTS * mag[clean], "rows that do not see it")
        du.assert_bf16(got[:, g:], want[:, g:], WEIGHTS * mag[:, g:], "other heads")
        if which == "v":                                            # infinities and NaN of values pass through their feature
            du.assert_bf16(got[sees][:, :g], want[sees][:, :g], np.nan_to_num(WEIGHTS * mag[sees][:, :g], posinf=0.0), "rows that see it")


def test_scores_of_every_size():
    """Rows whose maximum comes first or last, far above the others; scores near the largest number that is not infinite;
    a scale of 0 and a negative one."""
    b = _batch(9, [400, 130], [1, 9], 16, 4, 2, 128, std=8.0)
    for scale in (0.0, -0.05, 0.3, 1.0):
        _check(b, scale=scale)
    b.q *= 2.0**50
    b.k *= 2.0**40
    for i, (c, m) in enumerate(zip(b.context, b.fresh)):
        b.k[b.table[i, 3], 2] *= 4.0
    import decoder_util as du
    out, _ = _run(b, 1.0)
    want, _, mag = b.expected(1.0)
    du.assert_bf16(out, want, WEIGHTS * mag, "one key takes all")


def test_strided_tokens_and_outputs():
    from paper_2407_17029_amd import binding as qb
    b = _batch(10, [60, 3], [50, 1], 16, 8, 2, 128)
    a = b.device()
    ref = qb.qblora_paged_attention(**a, scale=0.1)
    joint = torch.zeros((b.T, 12, 128), dtype=torch.bfloat16, device=ref.device)
    joint[:, :8] = a["q"]
    a["q"] = joint[:, :8]
    out = torch.full((b.T, 10, 128), 7.0, dtype=torch.bfloat16, device=ref.device)
    qb.qblora_paged_attention(**a, scale=0.1, out=out[:, :8])
    torch.cuda.synchronize()
    assert torch.equal(out[:, :8], ref) and (out[:, 8:] == 7.0).all()


def test_repeats_its_bits_and_replays_in_a_graph():
    from paper_2407_17029_amd import binding as qb
    b = _batch(11, [900, 30, 2000], [40, 1, 1], 16, 8, 2, 128)
    a = b.device()
    kw = dict(scale=0.09, max_new=40)
    ws = torch.empty(qb.qblora_paged_attention_workspace_bytes(a["k_cache"], a["v_cache"], 8, 40), dtype=torch.uint8, device="cuda")
    ref = qb.qblora_paged_attention(**a, workspace=ws, **kw)
    again = qb.qblora_paged_attention(**a, **kw)
    torch.cuda.synchronize()
    assert torch.equal(ref, again)
    out = torch.zeros_like(ref)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            qb.qblora_paged_attention(**a, workspace=ws, out=out, **kw)
    for k in range(3):
        a["context"].copy_(torch.tensor([900 - k, 30, 2000 - 500 * k], dtype=torch.int32))   # lengths of another step
        out.fill_(3.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eager = qb.qblora_paged_attention(**a, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_cache_past_32_bit_offsets():
    """Pages on both sides of 2^31 elements."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    page, heads, dim = 256, 8, 256
    pages = (1 << 31) // (page * heads * dim) + 2
    small = _batch(12, [300, 200], [1, 30], page, heads, heads, dim)
    a = small.device()
    count = len(small.k)
    places = [0, pages - 1, pages - 2, 1, pages // 2, 2, 3][:count]
    kc = torch.zeros((pages,) + tuple(a["k_cache"].shape[1:]), dtype=torch.bfloat16, device=du.DEV)
    vc = torch.zeros((pages,) + tuple(a["v_cache"].shape[1:]), dtype=torch.bfloat16, device=du.DEV)
    for i, p in enumerate(places):
        kc[p], vc[p] = a["k_cache"][i], a["v_cache"][i]
    ref = qb.qblora_paged_attention(**a, scale=0.06)
    table = np.where(small.table >= 0, np.array(places)[np.maximum(small.table, 0)], -1)
    a.update(k_cache=kc, v_cache=vc, table=du.dev_i32(table))
    got = qb.qblora_paged_attention(**a, scale=0.06)
    torch.cuda.synchronize()
    assert torch.equal(ref, got)


def test_joins_of_prefixes_by_lse():
    """lse is what joins attention over two parts of a context: the result over both."""
    import decoder_util as du
    b = _batch(13, [150], [1], 16, 2, 2, 64)
    whole, lse = _run(b, 0.125)
    parts = []
    for cols in (slice(0, 4), slice(4, None)):
        t = b.table.copy()
        keep = np.zeros(t.shape[1], bool)
        keep[cols] = True
        t[:, ~keep] = -1
        full = b.table
        b.table = t
        parts.append([du.host(x) for x in _run(b, 0.125)])
        b.table = full
    w = [np.exp(p[1] - du.host(lse)) for p in parts]
    assert np.abs(w[0] + w[1] - 1.0).max() < 4e-4
    joined = parts[0][0] * w[0][..., None] + parts[1][0] * w[1][..., None]
    assert np.abs(joined - du.host(whole)).max() <= 3 * 2.0**-8 * np.abs(du.host(whole)).max()
