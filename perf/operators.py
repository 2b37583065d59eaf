"""What stands between the quantized projections of a decoder layer, as cases that can be timed and checked.

Four operators, each through the public binding:

  tables       block tables, slots and positions of the new tokens of a batch, made on the GPU from the requests' lengths
  rope_cache   rotary positions on q and k, and the rotated k and v written to a paged cache
  rope_train   rotary positions on q and k of a training batch, and the gradients' way back through them
  attn         attention of the new tokens of a batch (chunks, single tokens, or both) over a paged cache
  norm         addition of the residual and root-mean-square norm
  norm_train   the same with its backward pass

Head counts, widths and token counts are those of the LLaMA-shaped workloads in `paper_2407_17029_amd/synth.py` (32, 40 and
64 heads of 128; widths 4096, 5120, 8192), of `bench.py` and of the tests, or generic ones in between.

The paged cache holds, for each page and head, keys as [head_dim / 8, page, 8] and values as [page / 8, head_dim, 8]: eight
features of a position, or eight positions of a feature, lie together.  A slot is page_id * page + place in the page.

Lengths of a batch are drawn from the case (its "ragged" number), so that `work` knows them; values come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EPS = 1e-5


# ---- cases ----------------------------------------------------------------------------------------------

def listed():
    return [
        # One decoding step of 64 running requests: a token each, pages of 16.  The smallest call there is.
        dict(name="tables_decode_64", kind="tables", n=64, chunks=0, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=4096, page=16,
             ragged=1),
        # A large serving step: 1000 requests, 200 of them with a chunk of their prompt.
        dict(name="tables_mixed_1000", kind="tables", n=1000, chunks=200, new_lo=16, new_hi=1024, ctx_lo=0, ctx_hi=8192,
             page=32, ragged=2),
        # The same 64 single tokens in a 7B layer: latency.
        dict(name="rope_cache_7b_64", kind="rope_cache", n=64, chunks=0, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=4096, page=16,
             heads=32, kv_heads=32, dim=128, rot=128, layout="half", factor=1.0, packed=False, ragged=3),
        # Chunks of five prompts, 65B heads, in the product of one joint projection; adjacent pairs, long contexts.
        dict(name="rope_cache_65b_prompts", kind="rope_cache", n=5, chunks=5, new_lo=1200, new_hi=2100, ctx_lo=0, ctx_hi=60000,
             page=64, heads=64, kv_heads=64, dim=128, rot=128, layout="pairs", factor=8.0, packed=True, ragged=4),
        # A ragged training micro-batch of the 13B layer, both ways.
        dict(name="rope_train_13b_1337", kind="rope_train", T=1337, seq=512, heads=40, kv_heads=40, dim=128, rot=128,
             layout="half", factor=1.0),
        # Decoding one request of a 7B model: the cache of one context, latency.
        dict(name="attn_7b_1", kind="attn", n=1, chunks=0, new_lo=1, new_hi=1, ctx_lo=4095, ctx_hi=4095, page=16, heads=32,
             kv_heads=32, dim=128, window=0, ragged=5),
        # Decoding 64 requests of a 13B model with contexts of all lengths: the cache stream.
        dict(name="attn_13b_64", kind="attn", n=64, chunks=0, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=8000, page=16, heads=40,
             kv_heads=40, dim=128, window=0, ragged=6),
        # Four very long contexts, eight queries to a shared head.
        dict(name="attn_long_4", kind="attn", n=4, chunks=0, new_lo=1, new_hi=1, ctx_lo=30000, ctx_hi=131000, page=64,
             heads=64, kv_heads=8, dim=128, window=0, ragged=7),
        # A serving step with both: three chunks among single tokens, shared heads.
        dict(name="attn_mixed_16", kind="attn", n=16, chunks=3, new_lo=150, new_hi=512, ctx_lo=60, ctx_hi=4000, page=16,
             heads=64, kv_heads=8, dim=128, window=0, ragged=8),
        # A chunk of 4096 tokens of a long prompt in a 7B model: the largest call.
        dict(name="attn_7b_chunk_4096", kind="attn", n=1, chunks=1, new_lo=4096, new_hi=4096, ctx_lo=12288, ctx_hi=12288,
             page=64, heads=32, kv_heads=32, dim=128, window=0, ragged=9),
        # The norm before a 7B projection while decoding 64 requests.
        dict(name="norm_7b_64", kind="norm", T=64, d=4096, residual=True),
        # A full training batch of 8192 tokens at the 65B width, both ways.
        dict(name="norm_train_65b_8192", kind="norm_train", T=8192, d=8192, residual=True),
    ]


def draw(rng):
    """One more case of the same ranges."""

    def logint(lo, hi):
        v = min(hi, max(lo, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi + 0.5))))))
        return v | 1 if v > 2048 else v                             # large ones are odd

    kind = rng.choice(["tables", "rope_cache", "rope_train", "attn", "attn", "attn", "attn", "norm", "norm_train"])
    ragged = rng.randrange(1 << 30)
    if kind == "tables":
        n = logint(1, 2000)
        chunks = rng.choice([0, rng.randint(0, n)])
        hi = max(1, min(2048, 200000 // n))
        return dict(kind=kind, n=n, chunks=chunks, new_lo=1, new_hi=logint(1, hi), ctx_lo=0, ctx_hi=logint(16, 16000),
                    page=rng.choice([16, 32, 64, 128]), ragged=ragged)
    if kind in ("norm", "norm_train"):
        d = rng.choice([logint(500, 8192) | 1, (logint(32, 511) * 2 + 1) * 8])
        return dict(kind=kind, T=logint(1 if kind == "norm" else 64, 8192), d=d, residual=rng.random() < 0.8)
    dim = rng.choice([64, 128, 128, 128, 256])
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (64, 64), (64, 8), (32, 8), (40, 8), (16, 1), (12, 4), (7, 7)])
    if dim == 256:
        heads, kv_heads = rng.choice([(16, 16), (16, 4), (8, 1)])
    if kind.startswith("rope"):
        rot = rng.choice([dim, dim, dim // 2, dim // 4])
        rope = dict(heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, layout=rng.choice(["half", "pairs"]),
                    factor=rng.choice([1.0, 1.0, 4.0, 16.0]))
        if kind == "rope_train":
            return dict(kind=kind, T=logint(64, 8192), seq=logint(64, 4096), **rope)
        n = logint(1, 128)
        chunks = rng.choice([0, rng.randint(1, n)])
        hi = max(1, 8192 // max(1, chunks))
        return dict(kind=kind, n=n, chunks=chunks, new_lo=1, new_hi=logint(1, hi), ctx_lo=0, ctx_hi=logint(16, 60000),
                    page=rng.choice([16, 32, 64, 128]), packed=rng.random() < 0.5, ragged=ragged, **rope)
    form = rng.choice(["single", "single", "chunk", "mixed"])
    if form == "single":
        ctx = logint(32, 100000)
        n = logint(1, max(1, min(128, int(3e8 / (ctx * kv_heads * dim)))))
        return dict(kind=kind, n=n, chunks=0, new_lo=1, new_hi=1, ctx_lo=ctx // 8, ctx_hi=ctx, heads=heads, kv_heads=kv_heads,
                    dim=dim, page=rng.choice([16, 32, 64, 128]), window=rng.choice([0, 0, 0, logint(64, 4096)]), ragged=ragged)
    n = 1 if form == "chunk" else logint(2, 32)
    new = logint(8, max(8, min(4096, 16000 // n)))
    ctx = logint(16, max(16, min(16000, int(1.2e9 / (n * heads * new)))))
    return dict(kind=kind, n=n, chunks=1 if form == "chunk" else rng.randint(1, n), new_lo=max(1, new // 4), new_hi=new,
                ctx_lo=0, ctx_hi=ctx, heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([16, 32, 64, 128]),
                window=rng.choice([0, 0, 0, logint(64, 4096)]), ragged=ragged)


# ---- lengths --------------------------------------------------------------------------------------------

def lengths(case):
    """(tokens in the cache, new tokens) of each request; spread over the logarithm of their range."""
    r = random.Random(case["ragged"])

    def spread(lo, hi):
        v = min(hi, max(lo, int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** r.random() - 1))))
        return min(hi, v | 1) if v > 2048 else v

    fresh = [spread(case["new_lo"], case["new_hi"]) if i < case["chunks"] else 1 for i in range(case["n"])]
    context = [spread(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["n"])]
    r.shuffle(fresh)
    return context, fresh


def _pages(tokens, page):
    return -(-tokens // page)


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + stream) & (2**63 - 1))


def _normal(seed, stream, shape, std=1.0, dtype=BF16):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda", dtype=dtype).mul_(std)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _frequencies(rot, factor, original=4096):
    """Angle per position of each pair, in fp32, and the factor on q and k.  A context `factor` times as long as the
    original: pairs that turn often within it keep their frequency, those that turn less than once are slowed by the
    factor, the ones between are blended."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64) / rot)
    if factor == 1.0:
        return f.to(F32).cuda(), 1.0
    turns = original * f / (2.0 * math.pi)
    keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
    return (f * (keep + (1.0 - keep) / factor)).to(F32).cuda(), 0.1 * math.log(factor) + 1.0


def _cache(seed, pages, case):
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    return _normal(seed, 50, (pages, h, d // 8, page, 8)), _normal(seed, 51, (pages, h, page // 8, d, 8))


def prepare(case, seed):
    kind = case["kind"]
    st = {"kind": kind}
    if kind in ("norm", "norm_train"):
        T, d = case["T"], case["d"]
        st["x"], st["res"] = _normal(seed, 1, (T, d)), _normal(seed, 2, (T, d), 2.0) if case["residual"] else None
        st["w"] = (1.0 + _normal(seed, 3, (d,), 0.1, F32)).to(BF16)
        if kind == "norm_train":
            st["dy"], st["dsum"] = _normal(seed, 4, (T, d)), _normal(seed, 5, (T, d))
        return st
    if kind.startswith("rope"):
        st["freq"], st["scale"] = _frequencies(case["rot"], case["factor"])
        st["layout"] = case["layout"]
        h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if kind == "rope_train":
        T = case["T"]
        st["pos"] = torch.arange(T, device="cuda", dtype=torch.int32) % case["seq"]
        for i, name in enumerate(("q", "k", "dq", "dk")):
            st[name] = _normal(seed, i, (T, h if i % 2 == 0 else hk, d))
        return st

    context, fresh = lengths(case)
    n, page, total = case["n"], case["page"], sum(fresh)
    starts = [0]
    for m in fresh:
        starts.append(starts[-1] + m)
    have = [_pages(c, page) for c in context]
    want = [_pages(c + m, page) for c, m in zip(context, fresh)]
    held = have if kind == "tables" else want
    count = sum(want) + 7                                           # pages of the cache
    ids = torch.randperm(count, generator=_gen(seed, 60), device="cuda").to(torch.int32)
    # a row has space for what its request may grow to
    width = max(want) + 3
    cols = torch.arange(width, device="cuda")[None, :]
    first = torch.cumsum(_ints(held, torch.int64), 0) - _ints(held, torch.int64)
    at = (first[:, None] + cols).clamp(max=count - 1)
    table = torch.where(cols < _ints(held)[:, None], ids[at], -1).to(torch.int32)
    st["table"], st["context"] = table, _ints(context)
    if kind == "tables":
        st["fresh"], st["page"], st["free"] = _ints(fresh), page, ids[sum(held):].contiguous()
        st["tokens"] = -(-total // 64) * 64                         # a batch is padded to whole tiles
        return st
    st["starts"] = _ints(starts)
    if kind == "rope_cache":
        t = torch.arange(total, device="cuda")
        req = torch.repeat_interleave(torch.arange(n, device="cuda"), _ints(fresh, torch.int64), output_size=total)
        st["pos"] = (st["context"][req] + t - st["starts"][req]).to(torch.int32)
        st["slot"] = table[req, (st["pos"] // page).long()].long() * page + st["pos"] % page
        # only the pages that this step writes to: the others of a long context are not part of it
        used, inverse = torch.unique(torch.div(st["slot"], page, rounding_mode="floor"), return_inverse=True)
        st["slot"] = inverse * page + st["slot"] % page
        st["kc"], st["vc"] = _cache(seed, int(used.numel()), case)
        if case["packed"]:                                          # slices of one projection's output
            joint = _normal(seed, 10, (total, h + 2 * hk, d))
            st["q"], st["k"], st["v"] = joint[:, :h], joint[:, h:h + hk], joint[:, h + hk:]
        else:
            st["q"], st["k"], st["v"] = (_normal(seed, 10 + i, (total, c, d)) for i, c in enumerate((h, hk, hk)))
    else:
        st["kc"], st["vc"] = _cache(seed, count, case)
        st["q"] = _normal(seed, 10, (total, case["heads"], case["dim"]))
        st["window"], st["most"], st["longest"] = case["window"], max(fresh), max(c + m for c, m in zip(context, fresh))
    return st


# ---- the operators in plain form ------------------------------------------------------------------------

def _plain_tables(st):
    context, fresh, page, free, table = (st[k] for k in ("context", "fresh", "page", "free", "table"))
    n, width = table.shape
    have = (context + page - 1) // page
    want = ((context + fresh + page - 1) // page).clamp(max=width)
    more = (want - have).clamp(min=0)
    first = torch.cumsum(more, 0) - more
    col = torch.arange(width, device=table.device, dtype=torch.int32)[None, :]
    at = first[:, None] + col - have[:, None]
    ids = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table = torch.where((col >= have[:, None]) & (col < want[:, None]), ids, table).to(torch.int32)
    ends = torch.cumsum(fresh, 0).clamp(max=st["tokens"]).to(torch.int32)
    starts = torch.cat([torch.zeros_like(ends[:1]), ends])
    t = torch.arange(st["tokens"], device=table.device, dtype=torch.int32)
    req = torch.searchsorted(ends, t, right=True).clamp(max=n - 1)
    real = t < ends[-1]
    pos = torch.where(real, context[req] + t - starts[req], 0)
    place = pos // page
    page_id = table[req, place.clamp(max=width - 1).long()].long()
    slots = torch.where(real & (place < width) & (page_id >= 0), page_id * page + pos % page, -1)
    return {"table": table, "starts": starts, "positions": pos.to(torch.int32), "slots": slots,
            "taken": more.sum().reshape(1).to(torch.int32)}


def _turn(x, pos, freq, scale, layout, back=False):
    """Rotates the first 2 * len(freq) features of each head by position times frequency, in 32 bits."""
    angle = pos.to(F32)[:, None] * freq[None, :]
    c, s = (torch.cos(angle) * scale)[:, None, :], (torch.sin(angle) * (-scale if back else scale))[:, None, :]
    half = freq.numel()
    x32 = x.to(F32)
    turned, rest = x32[..., :2 * half], x32[..., 2 * half:]
    a, b = (turned[..., :half], turned[..., half:]) if layout == "half" else (turned[..., 0::2], turned[..., 1::2])
    u, v = a * c - b * s, b * c + a * s
    out = torch.cat([u, v], -1) if layout == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([out, rest], -1).to(x.dtype)


def _plain_norm(x, res, w):
    """The sum is rounded once, to the type it is kept in, and what is kept is normed."""
    total = (x.to(F32) + res.to(F32)).to(BF16).to(F32) if res is not None else x.to(F32)
    rstd = torch.rsqrt((total * total).mean(-1, keepdim=True) + EPS)
    return total, rstd, (total * rstd * w.to(F32)).to(BF16)


def _plain_norm_back(total, rstd, w, dy, dsum):
    hat = total.to(F32) * rstd
    g = dy.to(F32) * w.to(F32)
    dx = rstd * (g - hat * (g * hat).mean(-1, keepdim=True)) + dsum.to(F32)
    return dx.to(BF16), (dy.to(F32) * hat).sum(0)


def _plain_attn(st):
    q, kc, vc, table, starts, context = (st[k] for k in ("q", "kc", "vc", "table", "starts", "context"))
    T, heads, d = q.shape
    n, most, longest = context.numel(), st["most"], st["longest"]
    hk, page = kc.shape[1], kc.shape[3]
    pages = -(-longest // page)
    ids = table[:, :pages].clamp(min=0).long()
    # keys [n, hk, d, longest], values [n, hk, longest, d]
    k = kc[ids].to(F32).permute(0, 2, 3, 5, 1, 4).reshape(n, hk, d, pages * page)
    v = vc[ids].to(F32).permute(0, 2, 1, 3, 5, 4).reshape(n, hk, pages * page, d)
    j = torch.arange(most, device=q.device)
    fresh = (starts[1:] - starts[:-1])[:, None]
    row = (starts[:-1, None] + j[None, :]).clamp(max=T - 1)         # [n, most]
    x = q.to(F32)[row].reshape(n, most, hk, heads // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d)
    s = torch.matmul(x, k) / math.sqrt(d)
    here = context[:, None] + j[None, :]                            # position of each new token
    at = torch.arange(pages * page, device=q.device)[None, None, :]
    seen = (at <= here[:, :, None]) & (j[None, :, None] < fresh[:, :, None])
    if st["window"]:
        seen &= at > here[:, :, None] - st["window"]
    s = s.reshape(n, hk, heads // hk, most, -1).masked_fill_(~seen[:, None, None], float("-inf"))
    p = torch.exp_(s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)))
    p = p.div_(p.sum(-1, keepdim=True).clamp(min=1e-30)).reshape(n, hk, -1, pages * page)
    o = torch.matmul(p, v).reshape(n, hk, heads // hk, most, d).permute(0, 3, 1, 2, 4).reshape(n, most, heads, d)
    return o[(j[None, :] < fresh)].to(BF16)


def _plain(st):
    kind = st["kind"]
    if kind == "tables":
        return _plain_tables(st)
    if kind == "rope_train":
        turn = [(st[n], st["pos"], st["freq"], st["scale"], st["layout"]) for n in ("q", "k", "dq", "dk")]
        return {"q": _turn(*turn[0]), "k": _turn(*turn[1]), "dq": _turn(*turn[2], back=True), "dk": _turn(*turn[3], back=True)}
    if kind == "rope_cache":
        rope = (st["pos"], st["freq"], st["scale"], st["layout"])
        k, v, kc, vc = _turn(st["k"], *rope), st["v"], st["kc"], st["vc"]
        T, hk, d = k.shape
        page = kc.shape[3]
        p, o = torch.div(st["slot"], page, rounding_mode="floor"), st["slot"] % page
        kc[p, :, :, o] = k.reshape(T, hk, d // 8, 8)
        vc[p, :, o // 8, :, o % 8] = v
        return {"q": _turn(st["q"], *rope), "k": kc, "v": vc}
    if kind == "attn":
        return _plain_attn(st)
    total, rstd, y = _plain_norm(st["x"], st["res"], st["w"])
    out = {"y": y, "sum": total.to(BF16)} if st["res"] is not None else {"y": y}
    if kind == "norm_train":
        out["dx"], out["dw"] = _plain_norm_back(total, rstd, st["w"], st["dy"], st["dsum"])
    return out


def run(state):
    if not own:
        return _plain(state)
    from paper_2407_17029_amd import binding as qb
    st, kind = state, state["kind"]
    if kind == "tables":
        starts, pos, slots, taken = qb.qblora_page_tables(st["context"], st["fresh"], st["page"], st["free"], st["table"],
                                                          st["tokens"])
        return {"table": st["table"], "starts": starts, "positions": pos, "slots": slots, "taken": taken}
    if kind == "rope_train":
        pairs = st["layout"] == "pairs"
        q, k = qb.qblora_rope_fwd(st["q"], st["k"], st["pos"], st["freq"], interleaved=pairs, scale=st["scale"])
        dq, dk = qb.qblora_rope_bwd(st["dq"], st["dk"], st["pos"], st["freq"], interleaved=pairs, scale=st["scale"])
        return {"q": q, "k": k, "dq": dq, "dk": dk}
    if kind == "rope_cache":
        q = qb.qblora_rope_cache(st["q"], st["k"], st["v"], st["pos"], st["slot"], st["freq"], st["kc"], st["vc"],
                                 interleaved=st["layout"] == "pairs", scale=st["scale"])
        return {"q": q, "k": st["kc"], "v": st["vc"]}
    if kind == "attn":
        return qb.qblora_paged_attention(st["q"], st["kc"], st["vc"], st["table"], st["starts"], st["context"],
                                         1.0 / math.sqrt(st["q"].shape[2]), window=st["window"], max_new=st["most"])
    y, total, rstd = qb.qblora_rms_norm_fwd(st["x"], st["w"], EPS, residual=st["res"], keep=kind == "norm_train")
    out = {"y": y, "sum": total} if st["res"] is not None else {"y": y}
    if kind == "norm_train":
        out["dx"], out["dw"] = qb.qblora_rms_norm_bwd(total, st["w"], rstd, st["dy"], dtotal=st["dsum"])
    return out


# ---- the same from the definitions, in 64 bits ----------------------------------------------------------

def _turn64(x, pos, freq, scale, layout, sign):
    """Each pair as a complex number times exp(i * angle)."""
    half = freq.numel()
    z = torch.polar(torch.full((pos.numel(), half), scale, dtype=F64, device=x.device),
                    sign * pos.to(F64)[:, None] * freq.to(F64)[None, :])
    y = x.to(F64)
    if layout == "half":
        r = torch.complex(y[..., :half].contiguous(), y[..., half:2 * half].contiguous()) * z[:, None, :]
        y[..., :half], y[..., half:2 * half] = r.real, r.imag
    else:
        r = torch.complex(y[..., 0:2 * half:2].contiguous(), y[..., 1:2 * half:2].contiguous()) * z[:, None, :]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = r.real, r.imag
    return y


def _attn64(case, st):
    context, fresh = lengths(case)
    q, kc, vc = st["q"], st["kc"], st["vc"]
    T, heads, d = q.shape
    hk, page = case["kv_heads"], case["page"]
    out = torch.zeros((T, heads, d), dtype=F64, device=q.device)
    t0 = 0
    for i, (c, m) in enumerate(zip(context, fresh)):
        ids = st["table"][i, :_pages(c + m, page)].long()
        K = kc[ids].permute(1, 0, 3, 2, 4).reshape(hk, -1, d)[:, :c + m]
        V = vc[ids].permute(1, 0, 2, 4, 3).reshape(hk, -1, d)[:, :c + m]
        pos = torch.arange(c + m, device=q.device)
        for h in range(hk):
            rows = q[t0:t0 + m, h * (heads // hk):(h + 1) * (heads // hk)].to(F64)
            s = torch.matmul(rows.reshape(-1, d), K[h].to(F64).t().contiguous()) * d ** -0.5
            s = s.reshape(m, -1, c + m)
            for lo in range(0, m, 512):                             # some rows at a time
                part = s[lo:lo + 512]
                me = torch.arange(c + lo, c + lo + part.shape[0], device=q.device)[:, None, None]
                hide = pos[None, None, :] > me
                if case["window"]:
                    hide = hide | (pos[None, None, :] <= me - case["window"])
                part.masked_fill_(hide, float("-inf"))
            o = torch.matmul(torch.softmax(s, -1).reshape(-1, c + m), V[h].to(F64))
            out[t0:t0 + m, h * (heads // hk):(h + 1) * (heads // hk)] = o.reshape(m, -1, d)
        t0 += m
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "tables":
        return None                                                  # whole numbers
    if kind == "rope_train":
        return {n: _turn64(st[n], st["pos"], st["freq"], st["scale"], st["layout"], -1 if n[0] == "d" else 1)
                for n in ("q", "k", "dq", "dk")}
    if kind == "rope_cache":
        rope = (st["pos"], st["freq"], st["scale"], st["layout"], 1)
        kc, vc, k = st["kc"].to(F64), st["vc"].to(F64), _turn64(st["k"], *rope)
        pages, hk, d, page = kc.shape[0], case["kv_heads"], case["dim"], case["page"]
        flat = kc.permute(0, 3, 1, 2, 4).reshape(pages * page, hk, d)
        flat[st["slot"]] = k
        kc = flat.reshape(pages, page, hk, d // 8, 8).permute(0, 2, 3, 1, 4).contiguous()
        flat = vc.permute(0, 2, 4, 1, 3).reshape(pages * page, hk, d)
        flat[st["slot"]] = st["v"].to(F64)
        vc = flat.reshape(pages, page // 8, 8, hk, d).permute(0, 3, 1, 4, 2).contiguous()
        return {"q": _turn64(st["q"], *rope), "k": kc, "v": vc}
    if kind == "attn":
        return _attn64(case, st)
    x, w = st["x"].to(F64), st["w"].to(F64)
    both = x + st["res"].to(F64) if st["res"] is not None else x
    total = both.to(BF16).to(F64)                                    # as it is kept
    rms = torch.sqrt((total ** 2).sum(-1, keepdim=True) / case["d"] + EPS)
    out = {"y": total / rms * w}
    if st["res"] is not None:
        out["sum"] = both
    if kind == "norm_train":
        dy, unit = st["dy"].to(F64), total / rms
        g = dy * w
        out["dx"] = (g - unit * (g * unit).sum(-1, keepdim=True) / case["d"]) / rms + st["dsum"].to(F64)
        out["dw"] = (dy * unit).sum(0)
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_train"):
        e = case["T"] * case["d"]
        moved = 2.0 * e * (4 if case["residual"] else 2) + 2.0 * case["d"]
        flops = 5.0 * e
        if kind == "norm_train":                                    # sum, dy, dsum read; dx and dw written
            moved += 2.0 * e * 4 + 4.0 * case["d"]
            flops += 11.0 * e
        return {"bytes": moved, "flops": flops}
    if kind == "rope_train":
        e = case["T"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * 4.0 * e + 4.0 * case["T"], "flops": 2 * 3.0 * e * case["rot"] / case["dim"]}
    context, fresh = lengths(case)
    total, page = sum(fresh), case["page"]
    if kind == "tables":
        tokens = -(-total // 64) * 64
        more = sum(_pages(c + m, page) - _pages(c, page) for c, m in zip(context, fresh))
        return {"bytes": 12.0 * case["n"] + 4.0 + 8.0 * more + 12.0 * tokens, "flops": 4.0 * tokens}
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if kind == "rope_cache":
        return {"bytes": total * (4.0 * (h + 2 * hk) * d + 12.0), "flops": 3.0 * total * (h + hk) * case["rot"]}
    window = case["window"] or 1 << 40
    pairs = positions = 0
    for c, m in zip(context, fresh):
        positions += c + m - max(0, c + 1 - window)                  # seen by one row at least
        short = max(0, min(m, window - c))                           # rows whose window reaches the start
        pairs += short * c + short * (short + 1) // 2 + (m - short) * (window if m > short else 0)
    return {"bytes": 4.0 * positions * hk * d + 4.0 * total * h * d, "flops": 4.0 * pairs * h * d}
