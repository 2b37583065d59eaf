"""The operators between the projections on device-side integers that no plan would hold: nothing outside the buffers is
touched, and a call behind it is as ever."""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import WEIGHTS, _batch

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


def _guarded(count, dtype, inside):
    """(the whole buffer, its middle): `count` elements of `inside` between guards of 3."""
    buf = torch.full((count + 2 * GUARD,), 3, dtype=dtype, device="cuda")
    buf[GUARD:GUARD + count] = inside
    return buf, buf[GUARD:GUARD + count]


def _intact(buf):
    return bool((buf[:GUARD] == 3).all()) and bool((buf[-GUARD:] == 3).all())


@pytest.mark.parametrize("pattern", ["twice", "down", "wild"])
@pytest.mark.parametrize("n,T,heads,kv_heads,dim,max_new", [
    (6, 64, 8, 1, 64, 64),                                          # 72 units in a grid of 63, 12 of 12 tiles cut
    (40, 16, 1, 1, 128, 1),                                         # single tokens' form
    (6, 40, 4, 2, 256, 40), (80, 16, 2, 1, 64, 1), (80, 40, 8, 1, 128, 40),
])
def test_starts_that_do_not_ascend(n, T, heads, kv_heads, dim, max_new, pattern):
    """Tokens that several requests count as theirs make more units than the grid has.  What the workspace holds (here numbers far
    outside) is read for no tile that has not run."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    context, page = 3000, 64
    b = _batch(n + T, [context], [T], page, heads, kv_heads, dim, spare=0)
    a = b.device()
    good = du.dev_i32([0, T])
    starts = {"twice": [0, T] * n, "down": list(range(T, -n, -1)) + [0] * n, "wild": [0, T, -5, T + 9, 2**31 - 1, -2**31, 0, T] * n}[pattern][:n + 1]
    table, contexts = a["table"].expand(n, -1).contiguous(), du.dev_i32([context] * n)
    size = qb.qblora_paged_attention_workspace_bytes(a["k_cache"], a["v_cache"], heads, max_new)
    whole_ws, ws = _guarded(size, torch.uint8, 0x7f)
    whole, out = _guarded(T * heads * dim, torch.bfloat16, 9.0)
    whole_lse, lse = _guarded(T * heads, torch.float32, 9.0)
    out, lse = out.view(T, heads, dim), lse.view(T, heads)
    print(f"starts {pattern} n={n} T={T} heads={heads}/{kv_heads} dim={dim} max_new={max_new}", flush=True)
    kw = dict(scale=dim ** -0.5, max_new=max_new, workspace=ws)
    qb.qblora_paged_attention(a["q"], a["k_cache"], a["v_cache"], table, du.dev_i32(starts), contexts, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    assert _intact(whole) and _intact(whole_lse) and _intact(whole_ws)
    qb.qblora_paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], good, a["context"], out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    want, _, mag = b.expected(dim ** -0.5)
    du.assert_bf16(out, want, WEIGHTS * mag, "the call behind it")
