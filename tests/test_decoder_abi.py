"""The operators between the projections without a GPU: what their entry points refuse on the host and what they accept
without a launch, the sizes of their workspaces, rotary frequencies, and the gradient formulas that the GPU tests compare
with, against differences."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

import decoder_util as du

NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
A = 0x10000                                                # an address that is never read: the calls end before a launch
BIG = 1 << 40


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2407_17029_amd import build
        build.build_library()
    binding.lib()
    return binding


def cache(qb, **kw):
    f = dict(pages=100, page=64, heads=8, head_dim=128, k=A, v=A)
    f.update(kw)
    return qb.CKVCache(f["pages"], f["page"], f["heads"], f["head_dim"], f["k"], f["v"])


def check(call, defaults, cases):
    """Every case: what differs from a valid call, and the code it ends with."""
    for change, code in cases:
        assert not set(change) - set(defaults), change
        assert call(**{**defaults, **change}) == code, change


def test_page_tables(qb):
    order = ("context", "fresh", "n", "page", "free", "n_free", "table", "width", "tokens", "starts", "positions", "slots", "taken")
    good = dict(context=A, fresh=A, n=4, page=64, free=A, n_free=10, table=A, width=9, tokens=30, starts=A, positions=A, slots=A,
                taken=A)
    check(lambda **k: qb.lib().qblora_page_tables(*[k[x] for x in order], None), good, [
        (dict(n=-1), SHAPE), (dict(width=-1), SHAPE), (dict(tokens=-1), SHAPE), (dict(n_free=-1), SHAPE), (dict(page=0), SHAPE),
        (dict(page=-16), SHAPE), (dict(n=1 << 20, width=1 << 11), SHAPE), (dict(tokens=1 << 31), SHAPE),
        (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
    ] + [({name: None}, NULL) for name in ("context", "fresh", "free", "table", "starts", "positions", "slots", "taken")])


def rope(qb, rot=128, freq=A):
    return qb.CRope(rot, 0, 1.0, freq)


@pytest.mark.parametrize("name", ["qblora_rope_fwd", "qblora_rope_bwd"])
def test_rope(qb, name):
    order = ("rope", "q", "ldq", "heads", "k", "ldk", "kv_heads", "head_dim", "positions", "T", "q_out", "ldq_out", "k_out", "ldk_out")
    good = dict(rope=rope(qb), q=A, ldq=1024, heads=8, k=A, ldk=256, kv_heads=2, head_dim=128, positions=A, T=5, q_out=A,
                ldq_out=1024, k_out=A, ldk_out=256)

    def call(**k):
        return getattr(qb.lib(), name)(*[C.byref(k[x]) if x == "rope" and k[x] else k[x] for x in order], None)

    check(call, good, [
        (dict(rope=None), NULL), (dict(rope=rope(qb, freq=None)), NULL), (dict(q=None), NULL), (dict(positions=None), NULL),
        (dict(q_out=None), NULL), (dict(k_out=None), NULL),
        (dict(rope=rope(qb, rot=0)), SHAPE), (dict(rope=rope(qb, rot=127)), SHAPE), (dict(rope=rope(qb, rot=130)), SHAPE),
        (dict(rope=rope(qb, rot=-2)), SHAPE), (dict(T=-1), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
        (dict(head_dim=0), SHAPE), (dict(ldq=1023), SHAPE), (dict(ldk=255), SHAPE), (dict(ldq_out=1023), SHAPE), (dict(ldk_out=255), SHAPE),
        (dict(ldq=0), SHAPE), (dict(ldq=-1024), SHAPE), (dict(head_dim=1026, rope=rope(qb, rot=2)), UNSUPPORTED),
        (dict(heads=1 << 22, ldq=BIG, ldq_out=BIG), UNSUPPORTED), (dict(T=(1 << 30) + 1), UNSUPPORTED),
        (dict(T=0), 0), (dict(T=0, q=None, k=None, positions=None, q_out=None, k_out=None), 0),
        (dict(T=0, k=None, k_out=None, kv_heads=0, ldk=0, ldk_out=0), 0),
    ])


def test_rope_cache(qb):
    order = ("rope", "q", "ldq", "heads", "k", "ldk", "v", "ldv", "positions", "slots", "T", "q_out", "ldq_out", "cache")
    good = dict(rope=rope(qb), q=A, ldq=2048, heads=16, k=A, ldk=1024, v=A, ldv=1024, positions=A, slots=A, T=5, q_out=A, ldq_out=2048,
                cache=cache(qb))

    def call(**k):
        return qb.lib().qblora_rope_cache(*[C.byref(k[x]) if x in ("rope", "cache") and k[x] else k[x] for x in order], None)

    check(call, good, [({x: None}, NULL) for x in ("rope", "q", "k", "v", "positions", "slots", "q_out", "cache")] + [
        (dict(cache=cache(qb, k=None)), NULL), (dict(cache=cache(qb, v=None)), NULL),
        (dict(ldq=2047), SHAPE), (dict(ldk=1023), SHAPE), (dict(ldv=1023), SHAPE), (dict(ldq_out=2047), SHAPE), (dict(T=-1), SHAPE),
        (dict(heads=0), SHAPE), (dict(rope=rope(qb, rot=130)), SHAPE),
        (dict(cache=cache(qb, pages=0)), SHAPE), (dict(cache=cache(qb, heads=0)), SHAPE), (dict(cache=cache(qb, page=0)), SHAPE),
        (dict(cache=cache(qb, k=A + 8)), SHAPE), (dict(cache=cache(qb, v=A + 2)), SHAPE),
        (dict(cache=cache(qb, head_dim=96)), UNSUPPORTED), (dict(cache=cache(qb, head_dim=512)), UNSUPPORTED),
        (dict(cache=cache(qb, page=24)), UNSUPPORTED), (dict(cache=cache(qb, page=8)), UNSUPPORTED),
        (dict(T=0), 0), (dict(T=0, q=None, k=None, v=None, positions=None, slots=None, q_out=None), 0),
    ])


def test_paged_attention(qb):
    order = ("q", "ldq", "heads", "cache", "table", "width", "starts", "context", "n", "T", "scale", "window", "max_new", "out", "ldo",
             "lse", "workspace", "bytes")
    good = dict(q=A, ldq=2048, heads=16, cache=cache(qb), table=A, width=20, starts=A, context=A, n=3, T=7, scale=0.1, window=0,
                max_new=5, out=A, ldo=2048, lse=None, workspace=A, bytes=BIG)

    def call(**k):
        return qb.lib().qblora_paged_attention(*[C.byref(k[x]) if x == "cache" and k[x] else k[x] for x in order], None)

    need = qb.lib().qblora_paged_attention_workspace_bytes(C.byref(cache(qb)), 16, 5)
    check(call, good, [({x: None}, NULL) for x in ("q", "cache", "table", "starts", "context", "out")] + [
        (dict(n=-1), SHAPE), (dict(T=-1), SHAPE), (dict(width=-1), SHAPE), (dict(window=-1), SHAPE), (dict(max_new=-1), SHAPE),
        (dict(heads=0), SHAPE), (dict(heads=12, ldq=4096), SHAPE), (dict(ldq=2040), SHAPE), (dict(ldo=2040), SHAPE), (dict(ldq=2052), SHAPE),
        (dict(ldo=2052), SHAPE), (dict(q=A + 8), SHAPE), (dict(out=A + 2), SHAPE), (dict(workspace=A + 8), SHAPE),
        (dict(cache=cache(qb, pages=-1)), SHAPE), (dict(cache=cache(qb, k=A + 4)), SHAPE),
        (dict(cache=cache(qb, head_dim=80)), UNSUPPORTED), (dict(cache=cache(qb, page=40)), UNSUPPORTED),
        (dict(T=(1 << 30) + 1), UNSUPPORTED), (dict(width=1 << 25), UNSUPPORTED),
        (dict(workspace=None), WORKSPACE), (dict(bytes=need - 1), WORKSPACE),
        (dict(T=0), 0), (dict(n=0), 0), (dict(n=0, q=None, table=None, starts=None, context=None, out=None, workspace=None, bytes=0), 0),
    ])


def test_rms_norm(qb):
    L = qb.lib()
    f = ("x", "residual", "w", "T", "d", "eps", "total", "y", "rstd")
    check(lambda **k: L.qblora_rms_norm_fwd(*[k[x] for x in f], None),
          dict(x=A, residual=A, w=A, T=4, d=100, eps=1e-5, total=A, y=A, rstd=A),
          [({x: None}, NULL) for x in ("x", "w", "total", "y")] +
          [(dict(T=-1), SHAPE), (dict(d=0), SHAPE), (dict(d=-8), SHAPE), (dict(d=16385), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED),
           (dict(T=0), 0), (dict(T=0, x=None, residual=None, total=None, y=None, rstd=None), 0)])
    b = ("total", "w", "rstd", "dy", "dtotal", "T", "d", "dx", "dw", "workspace", "bytes")
    need = L.qblora_rms_norm_bwd_workspace_bytes(4, 100)
    check(lambda **k: L.qblora_rms_norm_bwd(*[k[x] for x in b], None),
          dict(total=A, w=A, rstd=A, dy=A, dtotal=A, T=4, d=100, dx=A, dw=A, workspace=A, bytes=need),
          [({x: None}, NULL) for x in ("total", "w", "rstd", "dy", "dx")] +
          [(dict(T=-1), SHAPE), (dict(d=0), SHAPE), (dict(workspace=A + 4), SHAPE), (dict(d=16385), UNSUPPORTED),
           (dict(workspace=None), WORKSPACE), (dict(bytes=need - 1), WORKSPACE),
           (dict(T=0, dw=None, total=None, rstd=None, dy=None, dx=None, workspace=None, bytes=0), 0)])


def test_workspace_sizes(qb):
    L = qb.lib()
    c = cache(qb)
    assert L.qblora_paged_attention_workspace_bytes(None, 8, 1) == 0
    assert L.qblora_paged_attention_workspace_bytes(C.byref(c), 12, 1) == 0                   # heads no multiple of 8
    one, few, many = [L.qblora_paged_attention_workspace_bytes(C.byref(c), 64, m) for m in (1, 4, 4096)]
    assert 0 < one <= few <= many < 1 << 30 and one % 16 == 0
    assert L.qblora_paged_attention_workspace_bytes(C.byref(c), 64, 1 << 20) == many          # no share of the tokens
    assert L.qblora_rms_norm_bwd_workspace_bytes(0, 100) == 0
    assert L.qblora_rms_norm_bwd_workspace_bytes(10, 20000) == 0
    sizes = [L.qblora_rms_norm_bwd_workspace_bytes(T, 1000) for T in (1, 5, 100, 10 ** 4, 10 ** 6)]
    assert sizes == sorted(sizes) and sizes[-1] <= 4096 * 4000


def test_the_binding_refuses(qb):
    """Types, shapes and layouts that a call could not describe: no pointer of such a tensor reaches the library."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        qb.qblora_rms_norm_fwd(x, w, 1e-5)                                                    # not on the device
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        qb.qblora_rope_fwd(q, None, i, torch.zeros(32))
    kc, vc = torch.zeros(3, 2, 8, 16, 8, dtype=torch.bfloat16), torch.zeros(3, 2, 2, 64, 8, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        qb.qblora_paged_attention(q, kc, vc, torch.zeros(1, 2, dtype=torch.int32), i[:2], i[:1], 0.1)
    with pytest.raises(AssertionError):
        qb.qblora_rope_cache(q, q, q, i, i.long(), torch.zeros(32), kc, vc)
    with pytest.raises(AssertionError):
        qb.qblora_page_tables(i, i, 16, i, torch.zeros(4, 2, dtype=torch.int32), 4, starts=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(qb.QBLoRAError):
        qb.qblora_rope_frequencies(7, device="cpu")
    with pytest.raises(qb.QBLoRAError):
        qb.qblora_rope_frequencies(8, kind=9, device="cpu")


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1e6)])
def test_frequencies(qb, rot, base):
    plain = [base ** (-2.0 * j / rot) for j in range(rot // 2)]
    factor, original, low, high = 4.0, 2048.0, 1.0, 32.0

    def want(kind):
        for f in plain:
            if kind == qb.ROPE_LINEAR:
                yield f / factor
            elif kind == qb.ROPE_BY_PARTS:
                g = min(max((original * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
                yield f * (g + (1 - g) / factor)
            else:
                yield f

    for kind in (qb.ROPE_PLAIN, qb.ROPE_LINEAR, qb.ROPE_BY_PARTS):
        got, scale = qb.qblora_rope_frequencies(rot, base, kind, factor, original, low, high, device="cpu")
        ref = np.array(list(want(kind)))
        assert got.dtype == torch.float32 and got.shape == (rot // 2,)
        assert (np.abs(got.numpy() - ref) <= 2.0 ** -23 * ref).all()                          # one rounding to 24 bits
        assert scale == np.float32(0.1 * math.log(factor) + 1.0 if kind == qb.ROPE_BY_PARTS else 1.0)
    if rot >= 4:
        got, scale = qb.qblora_rope_frequencies(rot, base, qb.ROPE_BASE, factor, device="cpu")
        assert scale == 1.0 and got[0] == 1.0
        assert abs(float(got[-1]) * factor / plain[-1] - 1.0) <= 2.0 ** -22                   # the slowest, slowed by the factor


def test_refused_frequencies(qb):
    out = (C.c_float * 64)()
    f = ("rot", "base", "kind", "factor", "original", "low", "high", "freq", "scale")
    good = dict(rot=128, base=1e4, kind=qb.ROPE_BY_PARTS, factor=2.0, original=4096.0, low=1.0, high=32.0, freq=out, scale=None)
    check(lambda **k: qb.lib().qblora_rope_frequencies(*[k[x] for x in f]), good, [
        ({}, 0), (dict(freq=None), NULL), (dict(rot=0), SHAPE), (dict(rot=5), SHAPE), (dict(base=0.0), SHAPE), (dict(base=math.nan), SHAPE),
        (dict(factor=0.0), SHAPE), (dict(factor=math.nan), SHAPE), (dict(original=0.0), SHAPE), (dict(low=32.0), SHAPE),
        (dict(rot=2, kind=qb.ROPE_BASE), SHAPE), (dict(kind=4), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED)])


# ---- the gradient formulas against differences -----------------------------------------------------------------------------

def differences(f, x, h=1e-5):
    """Central differences of a scalar function in every element of x."""
    out = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[at] += h
        down[at] -= h
        out[at] = (f(up) - f(down)) / (2 * h)
    return out


@pytest.mark.parametrize("d", [1, 2, 7, 32])
def test_norm_gradient_against_differences(d):
    """The loss sum(y * dy) + sum(total * dtotal) of a few rows: central differences are off by h^2 / 6 times the third
    derivative (rows of size one: a few units) and by the rounding of the loss, 1e-16 * d / h."""
    r = np.random.Generator(np.random.Philox(key=[d, 3]))
    total, dy, dtotal = r.standard_normal((3, 3, d))
    total += np.sign(total)                                                                  # no row next to zero
    w, eps = r.standard_normal(d) + 1.0, 1e-3

    def loss(total, w):
        return (du.norm(total, w, eps)[0] * dy).sum() + (total * dtotal).sum()

    dx, dw = du.norm_back(total, w, eps, dy, dtotal)
    assert np.abs(dx - differences(lambda t: loss(t, w), total)).max() <= 1e-8
    assert np.abs(dw - differences(lambda u: loss(total, u), w)).max() <= 1e-8


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,dim,rot", [(2, 8, 8), (1, 10, 4), (3, 2, 2)])
def test_rope_gradient_against_differences(heads, dim, rot, interleaved):
    """The operator is linear: differences are exact up to the rounding of the loss, 1e-16 * 100 / h."""
    r = np.random.Generator(np.random.Philox(key=[dim, 4]))
    x, dy = r.standard_normal((2, 4, heads, dim))
    positions, freq = np.array([0, 1, 77, 5000]), np.float32(0.5) ** np.arange(rot // 2, dtype=np.float32)

    def loss(x):
        return (du.rope(x, positions, freq, interleaved, 1.25) * dy).sum()

    dx = du.rope(dy, positions, freq, interleaved, 1.25, sign=-1.0)
    assert np.abs(dx - differences(loss, x)).max() <= 1e-8
