"""Sizes that the operators between the projections refuse on the host, as no grid or no 32-bit number holds them.  No GPU is needed:
the calls end before a launch."""
import ctypes as C

from test_decoder_abi import A, BIG, UNSUPPORTED, cache, qb  # noqa: F401


def test_attention_of_more_workgroups_than_a_grid_holds(qb):  # noqa: F811
    """Single tokens of 64 heads: a workgroup each at least, 2^24 of them 2^32 threads."""
    c = cache(qb, heads=64, head_dim=64)
    for n, max_new in ((1 << 18, 1), (1 << 17, 100), (1 << 20, 1)):
        rc = qb.lib().qblora_paged_attention(A, 64 * 64, 64, C.byref(c), A, 8, A, A, n, n, 0.1, 0, max_new, A, 64 * 64, None, A, BIG, None)
        assert rc == UNSUPPORTED, (n, max_new)


def test_tables_of_more_requests_than_their_arithmetic_holds(qb):  # noqa: F811
    """Requests are counted in groups, rounded up, in 32 bits."""
    for n, width in (((1 << 30) + 1, 1), (2**31 - 1, 1), (2**31 - 1, 0)):
        assert qb.lib().qblora_page_tables(A, A, n, 16, A, 4, A, width, 100, A, A, A, A, None) == UNSUPPORTED, (n, width)


def test_attention_of_more_requests_than_its_loops_count(qb):  # noqa: F811
    """They are taken 256 at a time, which passes 2^31 behind the last."""
    c = cache(qb)
    for n in ((1 << 30) + 1, 2**31 - 1):
        rc = qb.lib().qblora_paged_attention(A, 8 * 128, 8, C.byref(c), A, 0, A, A, n, 1, 0.1, 0, 1, A, 8 * 128, None, A, BIG, None)
        assert rc == UNSUPPORTED, n
