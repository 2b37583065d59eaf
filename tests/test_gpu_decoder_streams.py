"""The operators between the projections wait for the stream they are called on, and replay in a graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _normal(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)


def test_operators_read_what_a_busy_stream_has_yet_to_write():
    """Their inputs are NaN (and lengths and slots of nothing) until some milliseconds of products on a side stream are through."""
    from paper_2407_17029_amd import binding as qb
    n, T, heads, kv_heads, dim, page, d = 3, 40, 4, 2, 64, 16, 256
    f, _ = qb.qblora_rope_frequencies(dim)
    w, big = _normal(1, d), _normal(2, 8192, 8192)
    good_x, good_fresh = _normal(3, T, d), torch.tensor([1, 30, 9], dtype=torch.int32, device="cuda")
    x, fresh = torch.empty_like(good_x), torch.empty_like(good_fresh)
    context, free = torch.zeros_like(fresh), torch.arange(8, dtype=torch.int32, device="cuda")

    def run(chain):
        x.fill_(float("nan"))
        fresh.zero_()
        table = torch.full((n, 4), -1, dtype=torch.int32, device="cuda")
        kc = torch.zeros(8, kv_heads, dim // 8, page, 8, dtype=torch.bfloat16, device="cuda")
        vc = torch.zeros(8, kv_heads, page // 8, dim, 8, dtype=torch.bfloat16, device="cuda")
        torch.cuda.current_stream().synchronize()
        y = big
        for _ in range(chain):
            y = (big @ y).clamp(-1, 1)
        fresh.copy_(good_fresh)
        x.copy_(good_x)
        busy = chain and not torch.cuda.current_stream().query()
        y, _, rstd = qb.qblora_rms_norm_fwd(x, w, 1e-5, keep=True)
        dx, dw = qb.qblora_rms_norm_bwd(x, w, rstd, y)
        starts, p, slots, _ = qb.qblora_page_tables(context, fresh, page, free, table, T)
        q = y.view(T, heads, dim)
        a, b = qb.qblora_rope_fwd(q, q[:, :kv_heads], p, f)
        ga, gb = qb.qblora_rope_bwd(a, b, p, f)
        q = qb.qblora_rope_cache(q, b, b, p, slots, f, kc, vc)
        out = qb.qblora_paged_attention(q, kc, vc, table, starts, context, dim ** -0.5, max_new=30)
        return [y, rstd, dx, dw, table, starts, p, slots, a, b, ga, gb, kc, vc, out], busy

    run(1)                                                           # loads what the products take
    want, _ = run(0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, busy = run(20)
    side.synchronize()
    assert busy                                                      # the operators were issued before their inputs were there
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert all(torch.isfinite(t.float()).all() for t in want)


@pytest.mark.parametrize("T", [50, 1100])                            # rope and norm below and above the sizes of their other forms
def test_rope_and_norm_gradients_replay_in_a_graph(T):
    from paper_2407_17029_amd import binding as qb
    heads, kv_heads, dim, d = 48, 16, 128, 4096
    f, _ = qb.qblora_rope_frequencies(dim)
    w, p = _normal(1, d), torch.zeros(T, dtype=torch.int32, device="cuda")
    q, k, x, dy = (torch.zeros(*s, dtype=torch.bfloat16, device="cuda") for s in ((T, heads, dim), (T, kv_heads, dim), (T, d), (T, d)))

    def run():
        a, b = qb.qblora_rope_fwd(q, k, p, f)
        c, e = qb.qblora_rope_bwd(q, k, p, f)
        y, total, rstd = qb.qblora_rms_norm_fwd(x, w, 1e-5, residual=dy, keep=True)
        dx, dw = qb.qblora_rms_norm_bwd(total, w, rstd, dy, dtotal=x)
        only, _ = qb.qblora_rms_norm_bwd(total, w, rstd, dy, need_dw=False)
        return [a, b, c, e, y, total, rstd, dx, dw, only]

    run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs = run()
    for i in range(3):
        for j, t in enumerate((q, k, x, dy)):
            t.copy_(_normal(10 * i + j, *t.shape))
        p.copy_(torch.arange(T, device="cuda") * (i + 1) % 5000)
        for t in outs:
            t.fill_(3.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, run()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
