"""The weights of attention on few rows (single tokens, short runs of new ones) count with 16 bits: a row's output before it is stored
is off by at most 2^-16 of the weighted sum of |v| for the weights (bf16 of a weight, and bf16 of what that leaves: 2^-8 of 2^-8 each),
2e-5 for the scores as in test_gpu_paged_attention.py, and 4e-5 for fp32 sums of up to 700 terms (2^-24 of each partial sum)."""
import numpy as np
import pytest

from test_gpu_paged_attention import _batch, _run

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0**-16 + 2e-5 + 4e-5


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (8, 1, 64), (16, 2, 128), (4, 2, 256)])
@pytest.mark.parametrize("ctx,new,window", [([1, 2, 3, 7, 15, 16, 17, 31, 40, 100, 700], None, 0), ([30, 5, 600], None, 20), ([300, 8, 690], [2, 2, 2], 0)])
def test_outputs_of_few_rows(ctx, new, window, heads, kv_heads, dim):
    import decoder_util as du
    b = _batch(31 + dim + len(ctx), ctx, new or [1] * len(ctx), 16, heads, kv_heads, dim)
    out, _ = _run(b, dim ** -0.5, window, max_new=int(max(b.fresh)))
    want, _, mag = b.expected(dim ** -0.5, window)
    du.assert_bf16(out, want, WEIGHTS * mag, "out")


def test_long_contexts_in_parts():
    """9000 positions: the fp32 sums of each of 36 parts and of the join, 1.6e-5 and 2e-6 of the weighted sum."""
    import decoder_util as du
    b = _batch(32, [9000], [1], 64, 8, 2, 128)
    out, _ = _run(b, 128 ** -0.5, max_new=1)
    want, _, mag = b.expected(128 ** -0.5)
    du.assert_bf16(out, want, WEIGHTS * mag, "out")


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (8, 1, 64), (4, 2, 256)])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_values_that_are_not_finite_where_all_rows_see_them(heads, kv_heads, dim, bad):
    """In the middle of a context, where no mask is: infinities and NaN pass through their feature as the formula has it, with weights
    of every size, those that bf16 holds exactly (the largest is 1) among them."""
    import decoder_util as du
    b = _batch(33 + dim, [300, 90, 200], [1, 1, 2], 16, heads, kv_heads, dim)
    for i in range(3):
        for at, feature in ((5, 3), (40, 17), (70, 33)):
            b.v[b.table[i, at // 16], at % 16, 0, feature] = bad
        top = b.k[b.table[i, 2], 8, 0]                              # position 40 of every context has the largest weight
        top[:] = 4.0 * np.sign(b.q[b.starts[i], 0])
        b.q[b.starts[i]:b.starts[i + 1], :heads // kv_heads] = b.q[b.starts[i], 0]
    out, _ = _run(b, dim ** -0.5, max_new=2)
    want, _, mag = b.expected(dim ** -0.5)
    assert not np.isfinite(want[:, 0, [3, 17, 33]]).any()
    du.assert_bf16(out, want, np.nan_to_num(WEIGHTS * mag, posinf=0.0), "out")
