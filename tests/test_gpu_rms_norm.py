"""Residual addition and root-mean-square norm, both ways, against 64 bits.  The sum is bf16(x + residual), bit for bit.
y before it is stored: the mean of d squares in fp32 and three products, 1e-5 of the value.  dx: the same of each of its
terms.  dw: sums of T products in fp32, 8e-6 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _make(T, d, seed, residual=True, std=1.0):
    import decoder_util as du
    r = np.random.Generator(np.random.Philox(key=[seed, 41]))
    x = du.bf16(r.standard_normal((T, d)) * std)
    res = du.bf16(r.standard_normal((T, d)) * 2 * std) if residual else None
    w, dy, dt = (du.bf16(1.0 + 0.2 * r.standard_normal(d)), du.bf16(r.standard_normal((T, d))), du.bf16(r.standard_normal((T, d))))
    return x, res, w, dy, dt


def _total(x, res):
    import decoder_util as du
    return x if res is None else du.bf16((x.astype(np.float32) + res.astype(np.float32)))


SHAPES = [(1, 1), (3, 7), (5, 8), (2, 9), (64, 64), (33, 512), (7, 513), (64, 4096), (9, 4100), (5, 5120), (300, 96), (17, 8191),
          (16, 8192), (3, 8200), (2, 12001), (4, 16384), (3, 16383)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(T, d, residual):
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    x, res, w, _, _ = _make(T, d, T + d, residual)
    print(f"norm T={T} d={d}", flush=True)
    y, total, rstd = qb.qblora_rms_norm_fwd(du.dev_bf16(x), du.dev_bf16(w), EPS, residual=None if res is None else du.dev_bf16(res),
                                            keep=True)
    torch.cuda.synchronize()
    tot = _total(x, res)
    assert np.array_equal(du.host(total), tot)
    want, r = du.norm(tot, w, EPS)
    assert np.abs(host64(rstd) - r).max() <= 4e-6 * np.abs(r).max()
    du.assert_bf16(y, want, 1e-5 * np.abs(want), "y")


def host64(t):
    return t.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("T,d", SHAPES + [(2100, 40), (700, 1000)])
@pytest.mark.parametrize("with_dtotal", [True, False])
def test_backward(T, d, with_dtotal):
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    x, res, w, dy, dt = _make(T, d, 3 * T + d)
    tot = _total(x, res)
    dt = dt if with_dtotal else np.zeros_like(dt)
    total, wd = du.dev_bf16(tot), du.dev_bf16(w)
    print(f"norm backward T={T} d={d}", flush=True)
    _, _, rstd = qb.qblora_rms_norm_fwd(total, wd, EPS, keep=True)
    args = (total, wd, rstd, du.dev_bf16(dy))
    kw = dict(dtotal=du.dev_bf16(dt) if with_dtotal else None)
    dx, dw = qb.qblora_rms_norm_bwd(*args, **kw)
    torch.cuda.synchronize()
    want_x, want_w = du.norm_back(tot, w, EPS, dy, dt)
    r = 1.0 / np.sqrt((tot * tot).mean(-1, keepdims=True) + EPS)
    h, g = tot * r, dy * w
    du.assert_bf16(dx, want_x, 1e-5 * (r * (np.abs(g) + np.abs(h) * np.abs(g * h).mean(-1, keepdims=True)) + np.abs(dt)), "dx")
    assert (np.abs(host64(dw) - want_w) <= 8e-6 * np.abs(dy * h).sum(0) + 1e-30).all()
    dx2, dw2 = qb.qblora_rms_norm_bwd(*args, **kw)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)                   # repeated bits
    dx3, none = qb.qblora_rms_norm_bwd(*args, need_dw=False, **kw)
    torch.cuda.synchronize()
    assert none is None and torch.equal(dx, dx3)


def test_in_place():
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    x, res, w, dy, dt = _make(37, 1000, 9)
    xd, rd, wd = du.dev_bf16(x), du.dev_bf16(res), du.dev_bf16(w)
    y, total, rstd = qb.qblora_rms_norm_fwd(xd, wd, EPS, residual=rd, keep=True)
    dx, dw = qb.qblora_rms_norm_bwd(total, wd, rstd, du.dev_bf16(dy), dtotal=du.dev_bf16(dt))
    y2, total2, _ = qb.qblora_rms_norm_fwd(xd, wd, EPS, residual=rd, total=rd, y=xd)       # the stream and x are replaced
    d1, d2 = du.dev_bf16(dy), du.dev_bf16(dt)
    a, _ = qb.qblora_rms_norm_bwd(total, wd, rstd, d1, dtotal=d2, dx=d1)
    d1b = du.dev_bf16(dy)
    b, _ = qb.qblora_rms_norm_bwd(total, wd, rstd, d1b, dtotal=d2, dx=d2)
    torch.cuda.synchronize()
    assert y2.data_ptr() == xd.data_ptr() and torch.equal(y, y2) and torch.equal(total, total2)
    assert torch.equal(dx, a) and torch.equal(dx, b)


@pytest.mark.parametrize("d", [64, 100, 4096])
def test_unaligned_arrays(d):
    """Rows at any 2-byte address."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    x, res, w, dy, dt = _make(11, d, 4)

    def shifted(a, by):
        buf = torch.zeros(a.size + 16, dtype=torch.bfloat16, device=du.DEV)
        t = buf[by:by + a.size].view(a.shape)
        t.copy_(du.dev_bf16(a))
        return t

    ref = qb.qblora_rms_norm_fwd(du.dev_bf16(x), du.dev_bf16(w), EPS, residual=du.dev_bf16(res), keep=True)
    got = qb.qblora_rms_norm_fwd(shifted(x, 1), shifted(w, 3), EPS, residual=shifted(res, 5), keep=True,
                                 total=shifted(x, 7), y=shifted(x, 2))
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
    one = qb.qblora_rms_norm_bwd(ref[1], du.dev_bf16(w), ref[2], du.dev_bf16(dy), dtotal=du.dev_bf16(dt))
    two = qb.qblora_rms_norm_bwd(got[1], shifted(w, 1), got[2], shifted(dy, 3), dtotal=shifted(dt, 1), dx=shifted(dt, 9))
    torch.cuda.synchronize()
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_extreme_rows():
    """All zeros, the smallest and the largest values, infinities and NaN: what the formula gives in fp32."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    d = 256
    x = np.zeros((6, d))
    x[1] = 2.0**-60
    x[2] = 2.0**60                                             # the mean of squares is 2^120: still finite
    x[3, 5] = np.inf
    x[4, 7] = np.nan
    x[5] = np.random.default_rng(0).standard_normal(d)
    x = du.bf16(x)
    w = np.ones(d)
    y, _, rstd = qb.qblora_rms_norm_fwd(du.dev_bf16(x), du.dev_bf16(w), EPS, keep=True)
    torch.cuda.synchronize()
    got, r = du.host(y), host64(rstd)
    with np.errstate(invalid="ignore"):
        want, _ = du.norm(x, w, EPS)
    du.assert_bf16(got[[0, 1, 2, 5]], want[[0, 1, 2, 5]], 1e-5 * np.abs(want[[0, 1, 2, 5]]), "y")
    assert np.isnan(got[3, 5]) and (np.delete(got[3], 5) == 0).all()        # inf * 0, 0 elsewhere
    assert np.isnan(got[4]).all() and r[3] == 0.0


def test_no_rows():
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    w = du.dev_bf16(np.ones(100))
    e = torch.empty((0, 100), dtype=torch.bfloat16, device=du.DEV)
    qb.qblora_rms_norm_fwd(e, w, EPS, residual=e)
    dx, dw = qb.qblora_rms_norm_bwd(e, w, torch.empty(0, device=du.DEV), e)
    torch.cuda.synchronize()
    assert dx.shape == (0, 100) and (dw == 0).all()
