"""Rotary positions and norms of more rows than one launch takes (a grid has fewer than 2^32 threads): the bits of calls on parts."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _normal(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.bfloat16)


@pytest.mark.parametrize("dim,rot,interleaved", [(2, 2, False), (16, 16, True)])
def test_rope_of_many_tokens(dim, rot, interleaved):
    """2^24 tokens and some: a workgroup each."""
    from paper_2407_17029_amd import binding as qb
    T, part = (1 << 24) + 77, 1 << 20
    q, k = _normal(1, T, 1, dim), _normal(2, T, 1, dim)
    p = torch.arange(T, dtype=torch.int32, device="cuda")
    f, _ = qb.qblora_rope_frequencies(rot)
    print(f"rope T={T} dim={dim}", flush=True)
    for call in (qb.qblora_rope_fwd, qb.qblora_rope_bwd):
        whole = call(q, k, p, f, interleaved=interleaved)
        for i in range(0, T, part):
            a, b = call(q[i:i + part], k[i:i + part], p[i:i + part], f, interleaved=interleaved)
            assert torch.equal(whole[0][i:i + part], a) and torch.equal(whole[1][i:i + part], b), i


def test_rope_cache_of_many_tokens():
    """2^27 tokens of one head of 64, eight a workgroup, whose slots follow each other from within an octet."""
    from paper_2407_17029_amd import binding as qb
    T, dim, page = (1 << 27) + 21, 64, 256
    pages = T // page + 2
    x = _normal(3, T, 1, dim)
    p = torch.arange(T, dtype=torch.int32, device="cuda")
    slots = torch.arange(T, dtype=torch.int64, device="cuda") + 5
    f, _ = qb.qblora_rope_frequencies(dim)
    kc = torch.zeros(pages, 1, dim // 8, page, 8, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(pages, 1, page // 8, dim, 8, dtype=torch.bfloat16, device="cuda")
    print(f"rope_cache T={T}", flush=True)
    out = qb.qblora_rope_cache(x, x, x, p, slots, f, kc, vc)
    # around every place where a launch may end, and anywhere else; the rotated key is the rotated query, as both are x
    for at in [0, T // 3, T - 4096] + [(1 << b) - 2048 for b in range(20, 28)]:
        at = max(at, 0)
        n = min(4096, T - at)
        part, _ = qb.qblora_rope_fwd(x[at:at + n], None, p[at:at + n], f)
        assert torch.equal(out[at:at + n], part), at
        s = slots[at:at + n]
        assert torch.equal(kc[s // page, 0, :, s % page].reshape(n, 1, dim), part), at
        assert torch.equal(vc[s // page, 0, (s % page) // 8, :, s % 8].reshape(n, 1, dim), x[at:at + n]), at


@pytest.mark.parametrize("d", [3, 8])
def test_norm_of_many_rows(d):
    """2^26 rows and some of 64 threads each; the gradients' grid does not grow with the rows."""
    from paper_2407_17029_amd import binding as qb
    T, part = (1 << 26) + 9, 1 << 23
    x, r, w = _normal(4, T, d), _normal(5, T, d), _normal(6, d)
    print(f"norm T={T} d={d}", flush=True)
    y, total, rstd = qb.qblora_rms_norm_fwd(x, w, 1e-5, residual=r, keep=True)
    for i in range(0, T, part):
        a = qb.qblora_rms_norm_fwd(x[i:i + part], w, 1e-5, residual=r[i:i + part], keep=True)
        assert all(torch.equal(b[i:i + part], c) for b, c in zip((y, total, rstd), a)), i
    dx, _ = qb.qblora_rms_norm_bwd(total, w, rstd, y, need_dw=False)
    for i in (0, T // 2, T - 1000):
        assert torch.equal(dx[i:i + 1000], qb.qblora_rms_norm_bwd(total[i:i + 1000], w, rstd[i:i + 1000], y[i:i + 1000], need_dw=False)[0])
