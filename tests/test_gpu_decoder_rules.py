"""The operators between the projections on both sides of the rules that choose their forms, and on a stream of their own.

Rows (tokens) do not depend on one another in rotary positions and norms, and a form changes where results go and how work
is shared out, not the arithmetic of a row: a large call gives the bits of small ones.  Attention is compared with 64 bits
where contexts are cut in few and in many parts, in both of its forms."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import _batch, _check

pytestmark = pytest.mark.gpu


def _normal(seed, *shape):
    import decoder_util as du
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device=du.DEV, generator=g).to(torch.bfloat16)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T", [511, 512, 513, 1100])                         # 8 MB of results lie at 512 tokens
def test_large_rope_calls_give_the_bits_of_small_ones(T, interleaved):
    from paper_2407_17029_amd import binding as qb
    q, k = _normal(1, T, 48, 128), _normal(2, T, 16, 128)
    p = torch.arange(T, dtype=torch.int32, device="cuda") * 37 % 9001
    f, _ = qb.qblora_rope_frequencies(128)
    for call in (qb.qblora_rope_fwd, qb.qblora_rope_bwd):
        whole = call(q, k, p, f, interleaved=interleaved)
        parts = [call(q[i:i + 100], k[i:i + 100], p[i:i + 100], f, interleaved=interleaved) for i in range(0, T, 100)]
        for i in (0, 1):
            assert torch.equal(whole[i], torch.cat([x[i] for x in parts]))


@pytest.mark.parametrize("T,heads", [(255, 4), (256, 4), (257, 4), (600, 56), (1031, 8)])
@pytest.mark.parametrize("page", [16, 128])
def test_large_cache_calls_give_the_bits_of_small_ones(T, heads, page):
    """Tokens of two requests that follow each other, cut within octets of a page in the small calls."""
    from paper_2407_17029_amd import binding as qb
    kv_heads, dim = 4, 128
    q, k, v = _normal(3, T, heads, dim), _normal(4, T, kv_heads, dim), _normal(5, T, kv_heads, dim)
    fresh = torch.tensor([T // 3, T - T // 3], dtype=torch.int32, device="cuda")
    context = torch.tensor([5, 21], dtype=torch.int32, device="cuda")
    pages = T // page + 6
    table = torch.full((2, pages), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[1, :-(-21 // page)] = pages - 1, torch.arange(pages - 3, pages - 3 + -(-21 // page), dtype=torch.int32, device="cuda")
    free = torch.arange(pages - 3, dtype=torch.int32, device="cuda").flip(0).contiguous()
    _, p, slots, _ = qb.qblora_page_tables(context, fresh, page, free, table, T)
    assert int((slots < 0).sum()) == 0 and len(set(slots.tolist())) == T
    f, _ = qb.qblora_rope_frequencies(dim)

    def run(step):
        kc, vc = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")
                  for s in ((pages, kv_heads, dim // 8, page, 8), (pages, kv_heads, page // 8, dim, 8)))
        outs = [qb.qblora_rope_cache(*(t[i:i + step] for t in (q, k, v, p, slots)), f, kc, vc) for i in range(0, T, step)]
        return torch.cat(outs), kc, vc

    for a, b in zip(run(T), run(45)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1023, 1024, 1025])                            # 8 MB of results lie at 1024 rows
@pytest.mark.parametrize("residual", [False, True])
def test_large_norm_calls_give_the_bits_of_small_ones(T, residual):
    """dw: sums of T products in fp32, 8e-6 of the sum of magnitudes."""
    from paper_2407_17029_amd import binding as qb
    d = 4096
    x, r, dy, w = _normal(6, T, d), _normal(7, T, d) if residual else None, _normal(8, T, d), _normal(9, d)
    whole = qb.qblora_rms_norm_fwd(x, w, 1e-5, residual=r, keep=True)
    parts = [qb.qblora_rms_norm_fwd(x[i:i + 300], w, 1e-5, residual=None if r is None else r[i:i + 300], keep=True) for i in range(0, T, 300)]
    for i in range(3):
        assert torch.equal(whole[i], torch.cat([p[i] for p in parts]))
    total, rstd = whole[1], whole[2]
    dx, dw = qb.qblora_rms_norm_bwd(total, w, rstd, dy, dtotal=r)
    small = [qb.qblora_rms_norm_bwd(total[i:i + 300], w, rstd[i:i + 300], dy[i:i + 300], dtotal=None if r is None else r[i:i + 300])[0]
             for i in range(0, T, 300)]
    assert torch.equal(dx, torch.cat(small))
    terms = dy.double() * total.double() * rstd.double()[:, None]
    assert ((dw.double() - terms.sum(0)).abs() <= 8e-6 * terms.abs().sum(0)).all()


@pytest.mark.parametrize("ctx", [[511], [1023], [1024], [1025], [2047, 3], [4000], [9000], [9000, 0, 1]])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 128), (4, 2, 64), (16, 1, 256), (17, 1, 128)])
def test_single_tokens_in_parts(ctx, heads, kv_heads, dim):
    """From one part of a context to as many as there are, around the numbers that the join keeps in registers."""
    _check(_batch(len(ctx) + ctx[0], ctx, [1] * len(ctx), 16 if dim == 128 else 64, heads, kv_heads, dim))


@pytest.mark.parametrize("ctx,new,window", [
    ([4000], [17], 0), ([2100], [130], 0), ([2100, 0], [40, 3], 700), ([3000], [64], 2500), ([9, 1800], [5, 129], 0), ([0], [260], 0),
])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 128), (2, 1, 256), (3, 1, 64)])
def test_chunks_in_parts(ctx, new, window, heads, kv_heads, dim):
    _check(_batch(ctx[0] + new[0], ctx, new, 32, heads, kv_heads, dim), window=window)


def test_chunks_in_parts_with_pages_that_the_table_does_not_list():
    b = _batch(21, [2500, 64], [70, 33], 16, 2, 1, 128)
    b.table[0, 3:30] = -1
    b.table[0, 100] = 10 ** 6
    b.table[1, :4] = -5
    _check(b)
    _check(b, window=900)


def test_calls_on_another_stream():
    """Inputs made on a side stream, the operators behind them there, the results read there: nothing waits for, or runs
    on, the default stream."""
    from paper_2407_17029_amd import binding as qb
    n, heads, kv_heads, dim, page, d = 3, 4, 2, 64, 16, 256
    f, _ = qb.qblora_rope_frequencies(dim)
    ones = torch.ones(d, dtype=torch.bfloat16, device="cuda")

    def run():
        x = _normal(31, 40, d)
        for _ in range(20):                                                  # work that the operators have to wait for
            x = x.flip(0) * 1.0
        y, _, rstd = qb.qblora_rms_norm_fwd(x, ones, 1e-5, keep=True)
        dx, dw = qb.qblora_rms_norm_bwd(x, ones, rstd, y)
        fresh = torch.tensor([1, 30, 9], dtype=torch.int32, device="cuda")
        context = torch.zeros_like(fresh)
        table = torch.full((n, 4), -1, dtype=torch.int32, device="cuda")
        kc = torch.zeros(8, kv_heads, dim // 8, page, 8, dtype=torch.bfloat16, device="cuda")
        vc = torch.zeros(8, kv_heads, page // 8, dim, 8, dtype=torch.bfloat16, device="cuda")
        starts, p, slots, _ = qb.qblora_page_tables(context, fresh, page, torch.arange(8, dtype=torch.int32, device="cuda"), table, 40)
        q = y.view(40, heads, dim)
        k = v = q[:, :kv_heads]
        a, b = qb.qblora_rope_bwd(*qb.qblora_rope_fwd(q, k, p, f), p, f)
        q = qb.qblora_rope_cache(q, k, v, p, slots, f, kc, vc)
        out = qb.qblora_paged_attention(q, kc, vc, table, starts, context, dim ** -0.5, max_new=30)
        return [t.clone() for t in (y, dx, dw, table, a, b, kc, vc, out)]

    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert torch.isfinite(want[-1].float()).all()


@pytest.mark.parametrize("T,d", [(1, 70), (63, 513), (1024, 600), (1025, 600), (1000, 4096), (1024, 4096), (5, 16384)])
def test_norm_gradients_where_dy_is_replaced(T, d):
    """dx in a buffer of its own and in the place of dy: the same dx; dw within 8e-6 of the sum of magnitudes both times."""
    from paper_2407_17029_amd import binding as qb
    x, dy, w = _normal(10, T, d), _normal(11, T, d), _normal(12, d)
    _, total, rstd = qb.qblora_rms_norm_fwd(x, w, 1e-5, keep=True)
    terms = dy.double() * total.double() * rstd.double()[:, None]
    dx, dw = qb.qblora_rms_norm_bwd(total, w, rstd, dy)
    dx2, dw2 = qb.qblora_rms_norm_bwd(total, w, rstd, dy, dx=dy)
    assert dx2.data_ptr() == dy.data_ptr() and torch.equal(dx, dx2)
    for g in (dw, dw2):
        assert ((g.double() - terms.sum(0)).abs() <= 8e-6 * terms.abs().sum(0)).all()


@pytest.mark.parametrize("n,ctx,new", [(1, 900, 5), (3, 400, 8), (8, 120, 2), (20, 2100, 4), (64, 40, 3), (65, 40, 3), (70, 300, 8)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 1, 128), (16, 2, 64), (4, 1, 256)])
def test_a_few_tokens_of_several_requests(n, ctx, new, heads, kv_heads, dim):
    """17 to 64 rows of a request and fewer, in small batches and large ones, among single tokens and one chunk."""
    r = np.random.Generator(np.random.Philox(key=[n, new]))
    context = [int(x) for x in r.integers(0, ctx + 1, n)]
    fresh = [int(x) for x in r.integers(1, new + 1, n)]
    fresh[0] = new
    if n in (8, 65):
        fresh[n // 2] = 40
    _check(_batch(n + ctx, context, fresh, 16, heads, kv_heads, dim), window=100 if n == 3 else 0)


@pytest.mark.parametrize("T", [256, 300, 513])
@pytest.mark.parametrize("lengths", [[1], [1, 1, 1, 1, 9], [2, 3], [40, 1, 1]])
@pytest.mark.parametrize("page", [16, 64])
def test_many_tokens_of_short_runs_to_the_cache(T, lengths, page):
    """Slots that follow each other for so many tokens, then begin somewhere else; every seventeenth lies outside the cache.  The
    tolerance is that of test_gpu_rope.py."""
    import decoder_util as du
    from test_gpu_rope import _delta, _freq
    from paper_2407_17029_amd import binding as qb
    heads, kv_heads, dim = 3, 2, 64
    r = np.random.Generator(np.random.Philox(key=[T, len(lengths) + page]))
    pages = T // page * 2 + 8
    starts, slots, at = r.permutation(pages * page // 40) * 40, [], 0       # (a run is at most 40 long)
    while len(slots) < T:
        n = lengths[at % len(lengths)]
        slots += list(starts[at % len(starts)] + np.arange(n)) if at < len(starts) else [-1]
        at += 1
    slots = np.array(slots[:T], np.int64)
    slots[::17] = np.where(np.arange(len(slots[::17])) % 2, -3, pages * page + 5)
    q, k, v = (du.bf16(r.standard_normal((T, h, dim))) for h in (heads, kv_heads, kv_heads))
    p, f = r.integers(0, 100000, T).astype(np.int32), _freq(dim)
    kc0, vc0 = (du.bf16(r.standard_normal((pages, page, kv_heads, dim))) for _ in range(2))
    kc, vc = du.dev_bf16(du.key_pages(kc0)), du.dev_bf16(du.value_pages(vc0))
    got = qb.qblora_rope_cache(du.dev_bf16(q), du.dev_bf16(k), du.dev_bf16(v), du.dev_i32(p), torch.from_numpy(slots).to(du.DEV),
                               torch.from_numpy(f).to(du.DEV), kc, vc)
    torch.cuda.synchronize()
    du.assert_bf16(got, du.rope(q, p, f, False, 1.0), _delta(q, dim, False, 1.0), "q")
    inside = (slots >= 0) & (slots < pages * page)
    s = slots[inside]
    assert len(set(s.tolist())) == len(s)
    want_k, delta_k, want_v = kc0.copy(), np.zeros_like(kc0), vc0.copy()
    want_k[s // page, s % page] = du.rope(k, p, f, False, 1.0)[inside]
    delta_k[s // page, s % page] = _delta(k, dim, False, 1.0)[inside]
    want_v[s // page, s % page] = v[inside]
    du.assert_bf16(kc, du.key_pages(want_k), du.key_pages(delta_k), "keys")
    assert np.array_equal(du.host(vc), du.value_pages(want_v)), "values"


@pytest.mark.parametrize("seed", range(24))
def test_mixed_batches(seed):
    """Chunks, single tokens and idle requests of one batch, windows, pages that are not listed, a wrong max_new."""
    r = np.random.Generator(np.random.Philox(key=[seed, 77]))
    heads, kv_heads = [(4, 4), (8, 1), (6, 2), (16, 1), (20, 2), (8, 2)][seed % 6]
    dim, page = [64, 128, 256][seed % 3], [16, 32, 64, 256][seed % 4]
    n = [2, 5, 12, 66][seed // 6]
    context = [int(x) for x in r.integers(0, 400, n)]
    fresh = [int(x) for x in r.choice([0, 1, 1, 1, 4, 9] + [90] * (n < 20), n)]
    fresh[0] = 7
    b = _batch(seed, context, fresh, page, heads, kv_heads, dim)
    if seed % 5 == 0:
        b.table[r.random(b.table.shape) < 0.2] = [-1, 10 ** 6][seed % 2]
    _check(b, window=[0, 0, 33, 200][seed % 4], max_new=[None, max(fresh), 1][seed % 3])
