"""Rotary positions against 64-bit sines and cosines.  The kernel's value before it is stored is off by the hardware's sine
and cosine (within 1e-5 of 1) times the pair, and by an fp32 product: 1.5e-5 * scale * (|a| + |b|)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _inputs(T, heads, kv_heads, dim, seed, positions):
    import decoder_util as du
    r = np.random.Generator(np.random.Philox(key=[seed, 31]))
    q, k = du.bf16(r.standard_normal((T, heads, dim))), du.bf16(r.standard_normal((T, kv_heads, dim)))
    p = r.integers(0, positions, T).astype(np.int32)
    return q, k, p


def _freq(rot, base=10000.0):
    return (base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)


def _delta(x, rot, interleaved, scale):
    """1.5e-5 * scale * (|a| + |b|) for the features of pairs; the others are copied."""
    d = np.zeros_like(x)
    half = rot // 2
    i = np.arange(half)
    f0, f1 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    s = 1.5e-5 * scale * (np.abs(x[:, :, f0]) + np.abs(x[:, :, f1]))
    d[:, :, f0], d[:, :, f1] = s, s
    return d


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,heads,kv_heads,dim,rot,positions,scale", [
    (1, 32, 32, 128, 128, 4096, 1.0), (64, 7, 7, 128, 64, 100000, 1.2), (65, 8, 1, 64, 64, 64, 1.0),
    (9, 40, 8, 128, 32, 1 << 20, 0.7), (130, 3, 2, 256, 256, 2000, 1.0), (33, 2, 1, 256, 16, 2000, 1.0),
    (17, 5, 3, 80, 20, 500, 1.0),                            # a part that is no whole chunk
    (5, 3, 1, 6, 2, 50, 1.0), (4, 1, 1, 2, 2, 50, 1.0), (8, 2, 2, 96, 96, 300, 1.0), (300, 12, 4, 64, 16, 300, 1.0),
])
def test_forward_and_backward(T, heads, kv_heads, dim, rot, positions, scale, interleaved):
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    q, k, p = _inputs(T, heads, kv_heads, dim, T + dim, positions)
    f = _freq(rot)
    print(f"rope T={T} heads={heads}/{kv_heads} dim={dim} rot={rot}", flush=True)
    args = (du.dev_bf16(q), du.dev_bf16(k), du.dev_i32(p), torch.from_numpy(f).to(du.DEV))
    for call, sign in ((qb.qblora_rope_fwd, 1.0), (qb.qblora_rope_bwd, -1.0)):
        got = call(*args, interleaved=interleaved, scale=scale)
        torch.cuda.synchronize()
        for g, x, name in zip(got, (q, k), "qk"):
            du.assert_bf16(g, du.rope(x, p, f, interleaved, scale, sign), _delta(x, rot, interleaved, scale), f"{name} {sign}")


def test_backward_is_the_transposed_forward():
    """<turn(x), y> = <x, turn_back(y)>: each side's elements are rounded to bf16, 2^-9 of them at most."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    x, y, p = _inputs(50, 4, 4, 128, 3, 9000)
    f = torch.from_numpy(_freq(96)).to(du.DEV)
    a, _ = qb.qblora_rope_fwd(du.dev_bf16(x), None, du.dev_i32(p), f, scale=1.3)
    b, none = qb.qblora_rope_bwd(du.dev_bf16(y), None, du.dev_i32(p), f, scale=1.3)
    assert none is None
    left, right = du.host(a) * y, x * du.host(b)
    assert abs(left.sum() - right.sum()) <= 2.0**-8 * (np.abs(left).sum() + np.abs(right).sum()) / np.sqrt(left.size)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,offset,stride", [(20, 0, 12 * 128), (20, 4, 12 * 128 + 4), (3, 1, 12 * 128 + 3), (20, 8, 12 * 128 + 8)])
def test_strides_and_alignment(T, offset, stride, interleaved):
    """Slices of a joint projection at any 2-byte address and stride, into outputs with strides of their own, and in place."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    q, k, p = _inputs(T, 8, 4, 128, 5, 700)
    f = _freq(128)
    buf = torch.full((offset + T * stride,), float("nan"), dtype=torch.bfloat16, device=du.DEV)
    qs = buf.as_strided((T, 8, 128), (stride, 128, 1), offset)
    ks = buf.as_strided((T, 4, 128), (stride, 128, 1), offset + 8 * 128)
    qs.copy_(du.dev_bf16(q)); ks.copy_(du.dev_bf16(k))
    out = torch.full((offset + T * (stride + 2),), 7.0, dtype=torch.bfloat16, device=du.DEV)
    qo = out.as_strided((T, 8, 128), (stride + 2, 128, 1), offset)
    pos, freq = du.dev_i32(p), torch.from_numpy(f).to(du.DEV)
    _, ko = qb.qblora_rope_fwd(qs, ks, pos, freq, interleaved=interleaved, q_out=qo)
    torch.cuda.synchronize()
    want_q, want_k = du.rope(q, p, f, interleaved, 1.0), du.rope(k, p, f, interleaved, 1.0)
    du.assert_bf16(qo, want_q, _delta(q, 128, interleaved, 1.0), "q")
    du.assert_bf16(ko, want_k, _delta(k, 128, interleaved, 1.0), "k")
    beside = torch.ones_like(out, dtype=torch.bool)
    beside.as_strided((T, 8, 128), (stride + 2, 128, 1), offset).fill_(False)
    assert (out[beside] == 7.0).all()                          # nothing between the tokens is written
    qb.qblora_rope_fwd(qs, ks, pos, freq, interleaved=interleaved, q_out=qs, k_out=ks)
    torch.cuda.synchronize()
    assert torch.equal(qs, qo) and torch.equal(ks, ko)


def test_large_positions_keep_their_angle():
    """Near 2^31, where an fp32 angle knows nothing any more."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    q, k, _ = _inputs(40, 2, 1, 128, 8, 10)
    p = (2**31 - 1 - np.arange(40) * 977).astype(np.int32)
    f = _freq(128)
    got, _ = qb.qblora_rope_fwd(du.dev_bf16(q), du.dev_bf16(k), du.dev_i32(p), torch.from_numpy(f).to(du.DEV))
    du.assert_bf16(got, du.rope(q, p, f, False, 1.0), _delta(q, 128, False, 1.0), "q")


def _slots(r, runs, pages, page):
    """Slots of requests' runs of tokens: consecutive from any place, over pages in any order."""
    order, slots = r.permutation(pages), []
    at = 0
    for place, count in runs:
        need = -(-(place + count) // page)
        ids = order[at:at + need]
        at += need
        pos = place + np.arange(count)
        slots += list(ids[pos // page] * page + pos % page)
    return np.array(slots, np.int64)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,interleaved,runs", [
    (4, 4, 128, 128, False, [(0, 1), (5, 1), (15, 1), (8, 1)]),                   # single tokens
    (8, 2, 64, 32, True, [(0, 100)]), (3, 3, 128, 64, False, [(3, 61), (9, 7), (0, 8), (7, 2), (1, 1), (6, 30)]),
    (2, 1, 256, 256, True, [(13, 40), (0, 1), (8, 24)]), (32, 32, 128, 128, False, [(2, 3), (4, 1)]),
    (4, 4, 128, 128, True, [(1, 500)]), (2, 2, 64, 6, False, [(11, 77), (0, 9)]),
])
def test_cache_form(heads, kv_heads, dim, rot, interleaved, runs, page):
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    T = sum(c for _, c in runs)
    r = np.random.Generator(np.random.Philox(key=[T, page]))
    pages = sum(-(-(a + c) // page) for a, c in runs) + 2
    slots = _slots(r, runs, pages, page)
    q, k, p = _inputs(T, heads, kv_heads, dim, T, 5000)
    v = du.bf16(r.standard_normal((T, kv_heads, dim)))
    f = _freq(rot)
    kc0, vc0 = (du.bf16(r.standard_normal((pages, page, kv_heads, dim))) for _ in range(2))
    kc, vc = du.dev_bf16(du.key_pages(kc0)), du.dev_bf16(du.value_pages(vc0))
    print(f"rope_cache T={T} heads={heads}/{kv_heads} dim={dim} page={page}", flush=True)
    got = qb.qblora_rope_cache(du.dev_bf16(q), du.dev_bf16(k), du.dev_bf16(v), du.dev_i32(p), torch.from_numpy(slots).to(du.DEV),
                               torch.from_numpy(f).to(du.DEV), kc, vc, interleaved=interleaved, scale=1.1)
    torch.cuda.synchronize()
    du.assert_bf16(got, du.rope(q, p, f, interleaved, 1.1), _delta(q, rot, interleaved, 1.1), "q")
    want_k, delta_k, want_v = kc0.copy(), np.zeros_like(kc0), vc0.copy()
    want_k[slots // page, slots % page] = du.rope(k, p, f, interleaved, 1.1)
    delta_k[slots // page, slots % page] = _delta(k, rot, interleaved, 1.1)
    want_v[slots // page, slots % page] = v
    du.assert_bf16(kc, du.key_pages(want_k), du.key_pages(delta_k), "keys")
    assert np.array_equal(du.host(vc), du.value_pages(want_v)), "values"


def test_cache_form_writes_no_slot_outside():
    """Tokens without a page, slots behind the cache, and the neighbours of both."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    page, pages, heads, dim = 16, 3, 2, 64
    slots = np.array([-1, 0, 1, 2, 3, 4, 5, 6, 7, 8, -1, -1, 46, 47, 48, 49, 1 << 40, -(1 << 40), 20, -1], np.int64)
    T = len(slots)
    q, k, p = _inputs(T, 4, heads, dim, 77, 500)
    f = _freq(dim)
    guard = 4096
    size = pages * page * heads * dim
    bufs = [torch.full((size + 2 * guard,), 3.0, dtype=torch.bfloat16, device=du.DEV) for _ in range(2)]
    kc = bufs[0][guard:guard + size].view(pages, heads, dim // 8, page, 8)
    vc = bufs[1][guard:guard + size].view(pages, heads, page // 8, dim, 8)
    qb.qblora_rope_cache(du.dev_bf16(q), du.dev_bf16(k), du.dev_bf16(k), du.dev_i32(p), torch.from_numpy(slots).to(du.DEV),
                         torch.from_numpy(f).to(du.DEV), kc, vc)
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < pages * page)
    want_k, want_v = np.full((pages, page, heads, dim), 3.0), np.full((pages, page, heads, dim), 3.0)
    s = slots[ok]
    want_k[s // page, s % page] = du.rope(k, p, f, False, 1.0)[ok]
    want_v[s // page, s % page] = k[ok]
    delta = np.zeros_like(want_k)
    delta[s // page, s % page] = _delta(k, dim, False, 1.0)[ok]
    du.assert_bf16(kc, du.key_pages(want_k), du.key_pages(delta), "keys")
    assert np.array_equal(du.host(vc), du.value_pages(want_v))
    for b in bufs:
        assert (b[:guard] == 3.0).all() and (b[guard + size:] == 3.0).all()


def test_cache_past_32_bit_offsets():
    """A cache of more than 2^31 elements: slots on both sides."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    page, heads, dim = 256, 8, 256
    pages = (1 << 31) // (page * heads * dim) + 3
    slots = np.array([0, (pages - 3) * page - 1, (pages - 3) * page, pages * page - 1], np.int64)
    q, k, p = _inputs(4, 8, heads, dim, 5, 5000)
    f = _freq(dim)
    kc = torch.zeros((pages, heads, dim // 8, page, 8), dtype=torch.bfloat16, device=du.DEV)
    vc = torch.zeros((pages, heads, page // 8, dim, 8), dtype=torch.bfloat16, device=du.DEV)
    qb.qblora_rope_cache(du.dev_bf16(q), du.dev_bf16(k), du.dev_bf16(k), du.dev_i32(p), torch.from_numpy(slots).to(du.DEV),
                         torch.from_numpy(f).to(du.DEV), kc, vc)
    torch.cuda.synchronize()
    want = du.rope(k, p, f, False, 1.0)
    for i, s in enumerate(slots):
        got_k = kc[s // page, :, :, s % page].reshape(1, heads, dim)
        du.assert_bf16(got_k, want[i:i + 1], _delta(k[i:i + 1], dim, False, 1.0), f"key at slot {s}")
        got_v = vc[s // page, :, (s % page) // 8, :, s % 8].reshape(heads, dim)
        assert np.array_equal(du.host(got_v), k[i])
    count = int((kc != 0).sum())
    assert count <= 4 * heads * dim
