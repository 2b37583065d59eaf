"""The operators on many adapters and the optimizer's step without a GPU: what their entry points refuse and accept without a launch,
their sizes, and the formulas that the GPU tests compare with, against differences."""
import ctypes as C
import math
import os

import numpy as np
import pytest

import adapters_util as au

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


def adapters(qb, **kw):
    f = dict(count=5, d_in=512, d_out=256, lambda1=2, lambda2=4, R=32, table=A)
    f.update(kw)
    return qb.CAdapters(*(f[k] for k in ("count", "d_in", "d_out", "lambda1", "lambda2", "R", "table")))


BAD_ADAPTERS = [(dict(count=0), SHAPE), (dict(count=-1), SHAPE), (dict(count=8193), UNSUPPORTED), (dict(d_in=0), SHAPE),
                (dict(d_in=96), SHAPE), (dict(d_out=32), SHAPE), (dict(lambda1=0), SHAPE), (dict(lambda1=3), UNSUPPORTED),
                (dict(lambda2=16), UNSUPPORTED), (dict(lambda2=-2), SHAPE), (dict(R=0), SHAPE), (dict(R=12), SHAPE),
                (dict(R=520), UNSUPPORTED), (dict(table=None), NULL), (dict(table=A + 8), SHAPE), (dict(d_out=(1 << 20) + 64), UNSUPPORTED)]


def check(call, defaults, cases):
    """Every case: what differs from a valid call, and the code it ends with."""
    for change, code in cases:
        assert not set(change) - set(defaults), change
        assert call(**{**defaults, **change}) == code, change


def test_table(qb):
    def call(ads, first, n, list_, dA, dB):
        return qb.lib().qblora_adapter_table(C.byref(ads) if ads else None, first, n, list_, dA, dB, None)

    def entry(**kw):
        f = dict(l1=2, l2=4, R=32, s=1.0, A=A, B=A, op=0)
        f.update(kw)
        return (qb.CAdapter * 1)(qb.CAdapter(*(f[k] for k in ("l1", "l2", "R", "s", "A", "B", "op"))))

    at = lambda *p: (C.c_void_p * 1)(*p)  # noqa: E731
    good = dict(ads=adapters(qb), first=0, n=1, list_=entry(), dA=at(A), dB=at(A))
    check(call, good, [(dict(ads=adapters(qb, **c)), code) for c, code in BAD_ADAPTERS] + [
        (dict(ads=None), NULL), (dict(first=-1), SHAPE), (dict(n=-1), SHAPE), (dict(first=5), SHAPE), (dict(first=2, n=4), SHAPE),
        (dict(list_=None), NULL), (dict(dA=None), NULL), (dict(dB=None), NULL), (dict(dA=at(None)), NULL), (dict(dB=at(None)), NULL),
        (dict(list_=entry(l1=4)), SHAPE), (dict(list_=entry(l2=2)), SHAPE), (dict(list_=entry(R=40)), SHAPE),
        (dict(list_=entry(R=12)), SHAPE), (dict(list_=entry(R=-8)), SHAPE), (dict(list_=entry(op=1)), UNSUPPORTED),
        (dict(list_=entry(A=A + 8)), SHAPE), (dict(list_=entry(B=A + 2)), SHAPE), (dict(dA=at(A + 4)), SHAPE),
        (dict(n=0, list_=None), 0)])


def test_table_refuses_before_it_writes(qb):
    """The last entry of a long list is wrong: no launch has been made (there is no GPU here to make one on)."""
    ads = adapters(qb, count=100)
    entries = (qb.CAdapter * 100)(*[qb.CAdapter(2, 4, 32, 1.0, A, A, 0)] * 99, qb.CAdapter(2, 4, 33, 1.0, A, A, 0))
    assert qb.lib().qblora_adapter_table(C.byref(ads), 0, 100, entries, None, None, None) == SHAPE


def test_groups(qb):
    order = ("starts", "which", "n", "count", "T", "first", "order", "tiles")
    good = dict(starts=A, which=A, n=4, count=3, T=100, first=A, order=A, tiles=A)
    check(lambda **k: qb.lib().qblora_adapter_groups(*[k[x] for x in order], None), good, [
        (dict(n=-1), SHAPE), (dict(count=0), SHAPE), (dict(T=-1), SHAPE), (dict(n=8193), UNSUPPORTED), (dict(count=8193), UNSUPPORTED),
        (dict(T=(1 << 20) + 1), UNSUPPORTED), (dict(tiles=A + 4), SHAPE)] + [
        ({name: None}, NULL) for name in ("starts", "which", "first", "order", "tiles")])
    for count, T in ((1, 1), (3, 64), (3, 65), (500, 64), (8192, 1 << 20), (7, 0)):
        assert qb.lib().qblora_adapter_tiles(count, T) == au.tile_room(count, T)
    assert qb.lib().qblora_adapter_tiles(0, 5) == 0 and qb.lib().qblora_adapter_tiles(3, -5) == 0


@pytest.mark.parametrize("lengths", [[1] * 7, [64, 65, 1], [0, 0, 130], [63, 1, 64, 128, 129], [1000] + [1] * 30])
def test_tiles_fit_their_room(lengths):
    """Whatever the lengths of the adapters: runs of 64 need no more entries than there are."""
    T = sum(lengths)
    for count in (len(lengths), len(lengths) + 5):
        assert sum(-(-m // 64) for m in lengths) <= au.tile_room(count, T)


FWD = ("ads", "first", "order", "tiles", "X", "ldx", "T", "Y", "ldy", "saved", "ws", "ws_bytes")
BWD = ("ads", "first", "order", "tiles", "X", "ldx", "dY", "lddy", "T", "saved", "dX", "lddx", "gradients", "ws", "ws_bytes")


def test_forward(qb):
    def call(**k):
        return qb.lib().qblora_adapters_fwd(*[C.byref(k[x]) if x == "ads" and k[x] else k[x] for x in FWD], None)

    good = dict(ads=adapters(qb), first=A, order=A, tiles=A, X=A, ldx=512, T=10, Y=2 * A, ldy=256, saved=A, ws=A, ws_bytes=BIG)
    need = qb.lib().qblora_adapters_workspace_bytes(C.byref(good["ads"]), 10)
    assert need > 0 and need % 256 == 0
    check(call, good, [(dict(ads=adapters(qb, **c)), code) for c, code in BAD_ADAPTERS] + [
        (dict(ads=None), NULL), (dict(T=-1), SHAPE), (dict(T=(1 << 20) + 1), UNSUPPORTED), (dict(ldx=504), SHAPE), (dict(ldx=516), SHAPE),
        (dict(ldy=248), SHAPE), (dict(ldy=260), SHAPE), (dict(X=A + 8), SHAPE), (dict(Y=A + 2), SHAPE), (dict(saved=A + 8), SHAPE),
        (dict(tiles=A + 8), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=A + 16), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE),
        (dict(Y=A), SHAPE), (dict(T=0), 0), (dict(T=0, X=None, Y=None, order=None, tiles=None, ws=None, ws_bytes=0), 0)] + [
        ({name: None}, NULL) for name in ("first", "order", "tiles", "X", "Y")])


def test_backward(qb):
    def call(**k):
        return qb.lib().qblora_adapters_bwd(*[C.byref(k[x]) if x == "ads" and k[x] else k[x] for x in BWD], None)

    good = dict(ads=adapters(qb), first=A, order=A, tiles=A, X=A, ldx=512, dY=2 * A, lddy=256, T=10, saved=A, dX=3 * A, lddx=512, gradients=1, ws=A,
                ws_bytes=BIG)
    need = qb.lib().qblora_adapters_workspace_bytes(C.byref(good["ads"]), 10)
    check(call, good, [(dict(ads=adapters(qb, **c)), code) for c, code in BAD_ADAPTERS] + [
        (dict(T=-1), SHAPE), (dict(T=(1 << 20) + 1), UNSUPPORTED), (dict(ldx=508), SHAPE), (dict(lddy=252), SHAPE),
        (dict(lddx=500), SHAPE), (dict(X=A + 8), SHAPE), (dict(dY=A + 8), SHAPE), (dict(dX=A + 8), SHAPE), (dict(saved=A + 4), SHAPE),
        (dict(dX=None, gradients=0), NULL), (dict(dX=A), SHAPE), (dict(dX=2 * A), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE),
        (dict(T=0, gradients=0), 0), (dict(T=0, dX=None, gradients=0), NULL)] + [
        ({name: None}, NULL) for name in ("ads", "first", "order", "tiles", "X", "dY")])


def test_sizes(qb):
    L = qb.lib()
    a = adapters(qb, R=64)
    assert L.qblora_adapter_table_bytes(5) == 5 * 48 and L.qblora_adapter_table_bytes(0) == 0
    sizes = [L.qblora_adapters_saved_bytes(C.byref(a), T) for T in (0, 1, 100)]
    assert sizes[0] == 0 and sizes[2] == 100 * sizes[1] and sizes[1] >= 64 * 4
    assert [L.qblora_adapters_workspace_bytes(C.byref(a), T) for T in (-1, 0, (1 << 20) + 1)] == [0, 0, 0]
    # a workspace for the largest batch serves every smaller one
    for kw in (dict(), dict(count=1, d_in=13824, d_out=5120, R=256), dict(count=500, R=8), dict(count=3, d_in=64, d_out=64, R=512)):
        a = adapters(qb, **kw)
        sizes = [L.qblora_adapters_workspace_bytes(C.byref(a), T) for T in (*range(1, 1200), *range(1200, 60000, 37), 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    bad = adapters(qb, d_in=100)
    assert L.qblora_adapters_workspace_bytes(C.byref(bad), 10) == 0 and L.qblora_adapters_saved_bytes(None, 10) == 0


# ---- the optimizer's step ------------------------------------------------------------------------------------

def tensor(qb, **kw):
    f = dict(n=1000, param=A, master=A, grad=A, m=A, v=A, m_scale=A, v_scale=A, rate=1.0, decay=0.0)
    f.update(kw)
    return (qb.CAdamWTensor * 1)(qb.CAdamWTensor(*f.values()))


def test_plan(qb):
    def call(tensors, count, bits, plan, plan_bytes, out):
        return qb.lib().qblora_adamw_plan(tensors, count, bits, plan, plan_bytes, C.byref(out) if out else None, None)

    out = qb.CAdamWList()
    need = qb.lib().qblora_adamw_plan_bytes(tensor(qb), 1)
    good = dict(tensors=tensor(qb), count=1, bits=8, plan=A, plan_bytes=BIG, out=out)
    check(call, good, [
        (dict(count=-1), SHAPE), (dict(bits=16), UNSUPPORTED), (dict(tensors=None), NULL), (dict(plan=None), NULL), (dict(out=None), NULL),
        (dict(plan=A + 8), SHAPE), (dict(plan_bytes=need - 1), WORKSPACE)] + [
        (dict(tensors=tensor(qb, **{k: None})), NULL) for k in ("grad", "m", "v", "m_scale", "v_scale")] + [
        (dict(tensors=tensor(qb, param=None, master=None)), NULL), (dict(tensors=tensor(qb, n=-1)), SHAPE),
        (dict(tensors=tensor(qb, n=1 << 40)), SHAPE), (dict(tensors=tensor(qb, grad=A + 2)), SHAPE), (dict(tensors=tensor(qb, param=A + 1)), SHAPE),
        (dict(tensors=tensor(qb, master=A + 2)), SHAPE), (dict(tensors=tensor(qb, m_scale=A + 1)), SHAPE),
        (dict(bits=32, tensors=tensor(qb, m=A + 1)), SHAPE), (dict(tensors=tensor(qb, rate=math.nan)), SHAPE),
        (dict(tensors=tensor(qb, decay=math.inf)), SHAPE), (dict(count=0, tensors=None, plan=None, plan_bytes=0), 0)])
    assert out.count == 0 and out.bits == 8 and out.units == 0


def test_norm(qb):
    def call(list_, max_norm, out, ws, ws_bytes):
        return qb.lib().qblora_grad_norm(C.byref(list_) if list_ else None, max_norm, out, ws, ws_bytes, None)

    good = dict(list_=qb.CAdamWList(1, 32, 3, A), max_norm=1.0, out=A, ws=A, ws_bytes=BIG)
    need = qb.lib().qblora_grad_norm_workspace_bytes(C.byref(good["list_"]))
    assert need == 24
    check(call, good, [
        (dict(list_=None), NULL), (dict(list_=qb.CAdamWList(1, 32, 3, None)), NULL), (dict(list_=qb.CAdamWList(-1, 32, 3, A)), SHAPE),
        (dict(list_=qb.CAdamWList(1, 32, -3, A)), SHAPE), (dict(list_=qb.CAdamWList(1, 4, 3, A)), UNSUPPORTED),
        (dict(list_=qb.CAdamWList(1, 32, 3, A + 4)), SHAPE), (dict(out=None), NULL), (dict(max_norm=0.0), SHAPE),
        (dict(max_norm=-1.0), SHAPE), (dict(max_norm=math.nan), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE),
        (dict(ws=A + 8), WORKSPACE)])


def test_step(qb):
    def call(list_, how, clip):
        return qb.lib().qblora_adamw_step(C.byref(list_) if list_ else None, C.byref(how) if how else None, clip, None)

    def how(**kw):
        f = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, device_step=None, device_lr=None, seed=0)
        f.update(kw)
        return qb.CAdamW(*f.values())

    nothing = qb.CAdamWList(0, 8, 0, None)                  # a list without elements: no launch
    good = dict(list_=nothing, how=how(), clip=None)
    check(call, good, [
        ({}, 0), (dict(list_=None), NULL), (dict(how=None), NULL), (dict(list_=qb.CAdamWList(0, 7, 0, None)), UNSUPPORTED),
        (dict(how=how(beta1=1.0)), SHAPE), (dict(how=how(beta1=-0.1)), SHAPE), (dict(how=how(beta2=math.nan)), SHAPE),
        (dict(how=how(beta2=1.0)), SHAPE), (dict(how=how(beta2=1.0 - 1e-12)), SHAPE), (dict(how=how(eps=0.0)), SHAPE),
        (dict(how=how(eps=1e-60)), SHAPE), (dict(how=how(eps=9e-16)), SHAPE), (dict(how=how(eps=math.inf)), SHAPE), (dict(how=how(lr=math.nan)), SHAPE),
        (dict(how=how(step=0)), SHAPE), (dict(how=how(step=0, device_step=A)), 0), (dict(how=how(lr=math.nan, device_lr=A)), 0)])


# ---- the formulas that the GPU tests compare with --------------------------------------------------------------

def differences(f, x, h=1e-5):
    """Central differences of a scalar function in every element of x."""
    out = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[at] += h
        down[at] -= h
        out[at] = (f(up) - f(down)) / (2 * h)
    return out


@pytest.mark.parametrize("lam1,lam2", [(1, 1), (2, 2), (4, 1), (1, 8)])
def test_adapter_gradients_against_differences(lam1, lam2):
    """The loss sum(Y * dY) is linear in X, in every A and in every B: differences are exact up to its rounding, 1e-16 * 1000 / h."""
    b = au.Batch(3, 8, 8, lam1, lam2, [3, 2, 4], [2, 1, 0, 2], [1, 2, 0, 1], extra=1)

    def loss():
        return (b.forward()[0] * b.dY).sum()

    def with_(holder, key):
        def f(x):
            keep = holder[key]
            holder[key] = x
            try:
                return loss()
            finally:
                holder[key] = keep
        return f

    dX, dA, dB = b.backward()[:3]
    assert np.abs(dX - b.dX - differences(with_(vars(b), "X"), b.X)).max() <= 1e-7
    for a in range(3):
        assert np.abs(dA[a] - differences(with_(b.A, a), b.A[a])).max() <= 1e-7
        assert np.abs(dB[a] - differences(with_(b.B, a), b.B[a])).max() <= 1e-7
    assert not dA[0].any() and not dB[0].any() and np.array_equal(dX[-1], b.dX[-1])


def test_random_bits_are_even():
    """Of 2^18 elements each of the 32 bits is set in half, to five standard deviations (256 of 131072 each); so are the bits of
    neighbouring elements, tensors and steps together."""
    n = 1 << 18
    x = au.random_bits(n, 0, 7, 5)
    for y in (x, x[1:] ^ x[:-1], x ^ au.random_bits(n, 1, 7, 5), x ^ au.random_bits(n, 0, 8, 5), x ^ au.random_bits(n, 0, 7, 6),
              (x >> np.uint64(16)) ^ (x & np.uint64(0xffff)) | np.uint64(0xffff0000) & x):
        for bit in range(32):
            ones = int(((y >> np.uint64(bit)) & np.uint64(1)).sum())
            assert abs(ones - len(y) / 2) <= 5 * 0.5 * n ** 0.5, bit


def test_rounding_by_chance_keeps_the_mean():
    """A value rounded with all 2^16 random numbers: their mean is the value, to 2^-17 of the spacing (a random number counts as the
    middle of its sixteenth bit's step)."""
    r = np.arange(1 << 16, dtype=np.uint64)
    rng = np.random.Generator(np.random.Philox(key=[1, 1]))
    for a in list(rng.uniform(0, 448, 40)) + [1e-3, 2.0 ** -9, 0.0171, 2.0 ** -6, 447.9]:
        x = np.full(1 << 16, a)
        x[::256] = 448.0                                    # so that every block's scale is 1
        m, scale = au.Moments8._round(x, 448.0, 3, 2.0 ** -6, r, False)
        lower, upper = (v[0] for v in au.neighbours(np.array([a]), 3, 2.0 ** -6))
        rest = np.arange(1 << 16) % 256 != 0
        assert (scale == 1.0).all() and set(m[rest]) <= {lower, upper}
        part = (a - lower) / (upper - lower)
        assert abs((m[rest] == upper).mean() - part) <= 2.0 ** -16 + 2.0 ** -8      # a 256th of the random numbers is left out
