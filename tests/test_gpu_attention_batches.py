"""Attention on batches beyond those of the other tests: requests of 17 to 64 rows on both sides of the work that one wave of
workgroups takes, and tiles that are cut among more requests than a workgroup has threads."""
import numpy as np
import pytest

from test_gpu_attention_weights import WEIGHTS as FEW_WEIGHTS
from test_gpu_paged_attention import _batch, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,few", [(15, True), (40, False)])
def test_short_runs_in_small_and_large_batches(n, few):
    """32 rows a key head over 2080 to 2130 positions: two tiles of 16 rows, 66 or 67 blocks each, two key heads.  15 requests make at most
    4020 blocks, which is below the limit of 4096, 40 above 10500.  16 rows at a time, the weights count with 16 bits (and sums of
    2100 terms with 1.3e-4 at worst); in tiles of 128 with 8."""
    import decoder_util as du
    r = np.random.Generator(np.random.Philox(key=[n, 8]))
    b = _batch(n, [int(x) for x in r.integers(2080, 2127, n)], [4] * n, 64, 16, 2, 64)
    _check(b, max_new=4)
    if few:
        out, _ = _run(b, 0.125, max_new=4)
        want, _, mag = b.expected(0.125)
        du.assert_bf16(out, want, (FEW_WEIGHTS + 1e-4) * mag, "out")


@pytest.mark.parametrize("chunk", [0, 200])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 1, 64), (8, 4, 128), (2, 1, 256)])
def test_cut_tiles_among_many_requests(chunk, heads, kv_heads, dim):
    """Contexts of up to 3000 positions on both sides of the 256th request, among 600 short ones; with a chunk, more of them."""
    r = np.random.Generator(np.random.Philox(key=[chunk + dim, 9]))
    n = 600
    context, fresh = [int(x) for x in r.integers(0, 30, n)], [1] * n
    for at in (0, 3, 100, 255, 256, 257, 400, 511, 512, n - 1):
        context[at] = int(r.integers(1000, 3000))
    if chunk:
        for at in (2, 254, 258, 513):
            context[at], fresh[at] = int(r.integers(1500, 2500)), chunk if at == 258 else chunk // 4
    _check(_batch(n + dim, context, fresh, 16, heads, kv_heads, dim), max_new=chunk or 1)
