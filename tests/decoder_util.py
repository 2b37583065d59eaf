"""Plain 64-bit forms of the operators between the projections, and the tensors of their tests.

Everything here is numpy on the host, element by element from the definitions in include/qblora.h."""
import numpy as np
import torch

from paper_2407_17029_amd import synth

DEV = "cuda:0"


def bf16(x):
    """float array -> the bf16 values nearest to it, as float64."""
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


def dev_bf16(x):
    """float array (exact bf16 values or not) -> bf16 tensor on the device."""
    bits = synth.f32_to_bf16_bits(np.asarray(x, np.float32))
    return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).to(DEV)


def dev_i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ---- tables --------------------------------------------------------------------------------------------------

def tables(context, fresh, page, free, table, tokens):
    """(table, starts, positions, slots, taken) request by request."""
    table = table.copy()
    width = table.shape[1]
    starts, positions, slots, taken = [0], [], [], 0
    for i, (c, m) in enumerate(zip(context, fresh)):
        c, m = max(int(c), 0), max(int(m), 0)
        held, want = -(-c // page), min(-(-(c + m) // page), width)
        for col in range(held, want):
            table[i, col] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(c, c + m):
            positions.append(p)
            page_id = table[i, p // page] if p // page < width else -1
            slots.append(int(page_id) * page + p % page if page_id >= 0 else -1)
        starts.append(starts[-1] + m)
    pad = max(0, tokens - len(positions))
    positions = (positions + [0] * pad)[:tokens]
    slots = (slots + [-1] * pad)[:tokens]
    return table, np.minimum(starts, tokens), np.array(positions), np.array(slots), taken


# ---- rotary positions ----------------------------------------------------------------------------------------

def rope(x, positions, freq, interleaved, scale, sign=1.0):
    """x [T, heads, dim] float64, freq float32."""
    half = len(freq)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(freq, np.float64)[None, :]
    c, s = np.cos(angle)[:, None, :] * scale, sign * np.sin(angle)[:, None, :] * scale
    i = np.arange(half)
    f0, f1 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out = x.copy()
    out[:, :, f0] = x[:, :, f0] * c - x[:, :, f1] * s
    out[:, :, f1] = x[:, :, f1] * c + x[:, :, f0] * s
    return out


# ---- cache ---------------------------------------------------------------------------------------------------

def key_pages(k):
    """[pages, page, heads, dim] -> the layout of the cache."""
    pages, page, heads, dim = k.shape
    return np.ascontiguousarray(k.reshape(pages, page, heads, dim // 8, 8).transpose(0, 2, 3, 1, 4))


def value_pages(v):
    pages, page, heads, dim = v.shape
    return np.ascontiguousarray(v.reshape(pages, page // 8, 8, heads, dim).transpose(0, 3, 1, 4, 2))


# ---- attention -----------------------------------------------------------------------------------------------

def attention(q, k, v, table, starts, context, scale, window=0):
    """q [T, heads, dim], k and v [pages, page, kv_heads, dim], all float64 -> (out, lse, mag); rows of no request are NaN.
    mag: the weighted sum of |v| of each output, which rounding errors of the weights are relative to."""
    T, heads, dim = q.shape
    pages, page, kv_heads, _ = k.shape
    out, lse, mag = np.full((T, heads, dim), np.nan), np.full((T, heads), np.nan), np.zeros((T, heads, dim))
    for i in range(len(context)):
        for t in range(starts[i], starts[i + 1]):
            p = int(context[i]) + t - starts[i]
            lo = max(0, p - window + 1) if window else 0
            seen = np.arange(lo, p + 1)
            seen = seen[seen // page < table.shape[1]]
            ids = table[i, seen // page] if len(seen) else np.zeros(0, int)
            ok = (ids >= 0) & (ids < pages)
            seen, ids = seen[ok], ids[ok]
            for h in range(heads):
                if len(seen) == 0:
                    out[t, h], lse[t, h] = 0.0, -np.inf
                    continue
                K, V = k[ids, seen % page, h // (heads // kv_heads)], v[ids, seen % page, h // (heads // kv_heads)]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (K @ q[t, h])
                    top = s.max()
                    e = np.exp(s - top)
                    out[t, h] = (e[:, None] * V).sum(0) / e.sum()
                    mag[t, h] = (e[:, None] * abs(V)).sum(0) / e.sum()
                    lse[t, h] = top + np.log(e.sum())
    return out, lse, mag


class Batch:
    """A cache with the pages of `context` + `fresh` positions a request scattered over it, and what calls on it take.  What
    no request holds is NaN."""

    def __init__(self, seed, context, fresh, page, heads, kv_heads, dim, width=None, spare=3, std=1.0):
        r = np.random.Generator(np.random.Philox(key=[seed, 11]))
        self.context, self.fresh = np.array(context, np.int32), np.array(fresh, np.int32)
        self.starts = np.concatenate([[0], np.cumsum(self.fresh)]).astype(np.int32)
        self.T, self.page = int(self.starts[-1]), page
        need = [-(-(c + m) // page) for c, m in zip(context, fresh)]
        pages = sum(need) + spare
        width = max(need + [1]) + 2 if width is None else width
        order = r.permutation(pages)
        self.table = np.full((len(context), width), -1, np.int32)
        self.k = np.full((pages, page, kv_heads, dim), np.nan)
        self.v = np.full((pages, page, kv_heads, dim), np.nan)
        at = 0
        for i, (c, m) in enumerate(zip(context, fresh)):
            ids = order[at:at + need[i]]
            at += need[i]
            self.table[i, :min(need[i], width)] = ids[:width]
            pos = np.arange(c + m)
            self.k[ids[pos // page], pos % page] = bf16(r.standard_normal((c + m, kv_heads, dim)))
            self.v[ids[pos // page], pos % page] = bf16(r.standard_normal((c + m, kv_heads, dim)))
        self.q = bf16(r.standard_normal((self.T, heads, dim)) * std)

    def device(self):
        return dict(q=dev_bf16(self.q), k_cache=dev_bf16(key_pages(self.k)), v_cache=dev_bf16(value_pages(self.v)),
                    table=dev_i32(self.table), starts=dev_i32(self.starts), context=dev_i32(self.context))

    def expected(self, scale, window=0):
        return attention(self.q, self.k, self.v, self.table, self.starts, self.context, scale, window)


# ---- root-mean-square norm -----------------------------------------------------------------------------------

def norm(total, w, eps):
    """(y, rstd) of rows in float64."""
    rstd = 1.0 / np.sqrt((total * total).mean(-1) + eps)
    return total * rstd[:, None] * w, rstd


def norm_back(total, w, eps, dy, dtotal):
    rstd = 1.0 / np.sqrt((total * total).mean(-1, keepdims=True) + eps)
    h, g = total * rstd, dy * w
    return rstd * (g - h * (g * h).mean(-1, keepdims=True)) + dtotal, (dy * h).sum(0)


# ---- comparison ----------------------------------------------------------------------------------------------

def half_step(x):
    """Half the spacing of bf16 numbers at |x|."""
    a = np.abs(x)
    with np.errstate(invalid="ignore"):
        e = np.floor(np.log2(np.where((a > 0) & np.isfinite(a), a, 1.0)))
    return np.where(a > 0, np.exp2(e - 8.0), 0.0)


def assert_bf16(got, ref, delta, what):
    """A value that is within `delta` of ref before it is rounded to bf16: at most delta plus half a spacing off.  NaN and
    infinities where the reference has them and nowhere else."""
    g = host(got) if isinstance(got, torch.Tensor) else got
    delta = np.broadcast_to(delta, ref.shape)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(g), np.isnan(ref)), f"{what}: NaN elsewhere"
    assert np.array_equal(g[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), f"{what}: infinities elsewhere"
    if not fine.any():
        return
    allowed = (delta + half_step(np.abs(ref) + delta))[fine]
    err = np.abs(g[fine] - ref[fine])
    worst = np.argmax(err - allowed)
    assert (err <= allowed).all(), f"{what}: off by {err[worst]:.3e} where {allowed[worst]:.3e} is allowed, at {ref[fine][worst]:.3e}"
