"""Many adapters on one frozen projection, served and trained, as cases that can be timed and checked.

Four operators, each through the public binding:

  groups   the tokens of a batch grouped by the adapter of their request
  serve    the adapter terms of a batch, each request's with its own adapter, added to the shared projection's output
  train    the same with its backward pass: gradients of the inputs and of every adapter's matrices
  adamw    one AdamW step over many tensors, with the norm of all gradients and its clipping in front of it

Layer shapes are those of the LLaMA-shaped workloads in `paper_2407_17029_amd/synth.py` (widths 4096, 5120, 8192 with 11008, 13824,
22016; inner rank R = lambda * rank with rank 64 or 128), of the tests, or generic ones in between.

For token t of a request with adapter a, C the mean of `lam1` adjacent inputs and E the repetition of each value `lam2` times:

  Y[t] += s_a * E(C(X[t]) A_a B_a)

A request without adapter (-1) leaves its rows as they are.  Adapters, lengths and ranks of a batch are drawn from the case (its
"ragged" number), so that `work` knows them; values come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
TILE = 64                                                            # tokens of a tile at most


# ---- cases ----------------------------------------------------------------------------------------------

def _proj(d_in, d_out, lam, R):
    return dict(d_in=d_in, d_out=d_out, lam1=lam, lam2=lam, R=R)


def listed():
    return [
        # One decoding step of 64 running requests on 16 loaded adapters, once for all projections.  The smallest call.
        dict(name="groups_decode_64", kind="groups", n=64, chunks=0, new_lo=1, new_hi=1, count=16, bare=0.1, ragged=1),
        # A large serving step: 1000 requests, 200 of them with a chunk of their prompt, 500 adapters.
        dict(name="groups_mixed_1000", kind="groups", n=1000, chunks=200, new_lo=16, new_hi=1024, count=500, bare=0.1, ragged=2),
        # Eight single tokens, eight adapters of a 7B attention projection: latency.
        dict(name="serve_7b_8", kind="serve", n=8, chunks=0, new_lo=1, new_hi=1, count=8, bare=0.0, mixed=False, ragged=3,
             **_proj(4096, 4096, 2, 128)),
        # 64 single tokens over 40 adapters of several ranks on a 7B gate projection: the stream of the adapters.
        dict(name="serve_7b_gate_64", kind="serve", n=64, chunks=0, new_lo=1, new_hi=1, count=40, bare=0.1, mixed=True, ragged=4,
             **_proj(4096, 11008, 2, 128)),
        # 256 single tokens over 100 adapters on a 65B gate projection.
        dict(name="serve_65b_gate_256", kind="serve", n=256, chunks=0, new_lo=1, new_hi=1, count=100, bare=0.05, mixed=False,
             ragged=5, **_proj(8192, 22016, 2, 256)),
        # A serving step with both: eight chunks of prompts among single tokens, 13B down projection.
        dict(name="serve_13b_down_mixed", kind="serve", n=24, chunks=8, new_lo=150, new_hi=1500, count=12, bare=0.1, mixed=True,
             ragged=6, **_proj(13824, 5120, 2, 128)),
        # A small training batch of 16 adapters with larger tiles (lambda 4), ragged sequences.
        dict(name="train_7b_16", kind="train", n=24, chunks=24, new_lo=20, new_hi=130, count=16, bare=0.0, mixed=True, ragged=7,
             **_proj(4096, 4096, 4, 64)),
        # Four adapters trained side by side on a 7B attention projection, a full batch of about 8192 tokens.
        dict(name="train_7b_4", kind="train", n=16, chunks=16, new_lo=400, new_hi=620, count=4, bare=0.0, mixed=False, ragged=8,
             **_proj(4096, 4096, 2, 128)),
        # Two adapters on a 65B up projection, about 8192 tokens: the largest call of them.
        dict(name="train_65b_up_2", kind="train", n=8, chunks=8, new_lo=900, new_hi=1100, count=2, bare=0.0, mixed=False, ragged=9,
             **_proj(8192, 22016, 2, 256)),
        # Three small adapters of odd rank and their norms' weights: latency.
        dict(name="adamw8_small", kind="adamw", bits=8, tensors=9, lo=37, hi=40000, layers=0, master=True, clip=True, ragged=10),
        # All adapters of a 7B layer (14 matrices, 5 million elements), states in 32 bits.
        dict(name="adamw32_7b_layer", kind="adamw", bits=32, tensors=0, lo=0, hi=0, layers=1, master=True, clip=True, ragged=7),
        # All adapters of six 65B layers (84 matrices, 120 million elements), states in 8 bits.
        dict(name="adamw8_65b_layers", kind="adamw", bits=8, tensors=0, lo=0, hi=0, layers=6, master=True, clip=True, ragged=65),
    ]


_SHAPES = [(4096, 4096), (4096, 11008), (11008, 4096), (5120, 5120), (5120, 13824), (13824, 5120), (8192, 8192), (8192, 22016),
           (22016, 8192), (512, 512), (1024, 2048), (2048, 640)]


def draw(rng):
    """One more case of the same ranges."""

    def logint(lo, hi):
        v = min(hi, max(lo, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi + 0.5))))))
        return v | 1 if v > 2048 else v                             # large ones are odd

    kind = rng.choice(["groups", "serve", "serve", "serve", "train", "train", "adamw", "adamw"])
    ragged = rng.randrange(1 << 30)
    bare = rng.choice([0.0, 0.1, 0.5])
    if kind == "groups":
        n = logint(2, 2000)
        hi = max(1, min(2048, 200000 // n))
        return dict(kind=kind, n=n, chunks=rng.choice([0, rng.randint(0, n)]), new_lo=1, new_hi=logint(1, hi), count=logint(2, 1000),
                    bare=bare, ragged=ragged)
    if kind == "adamw":
        form = rng.choice(["layers", "odd", "odd"])
        return dict(kind=kind, bits=rng.choice([8, 32]), tensors=0 if form == "layers" else logint(1, 300), lo=1,
                    hi=logint(100, 300000), layers=rng.randint(1, 3) if form == "layers" else 0, master=rng.random() < 0.7,
                    clip=rng.random() < 0.5, ragged=ragged)
    d_in, d_out = rng.choice(_SHAPES)
    lam = rng.choice([1, 2, 2, 4, 8])
    R = rng.choice([8, 16, 32, 64, 64, 128, 128, 256])
    both = dict(kind=kind, bare=bare, mixed=rng.random() < 0.5, ragged=ragged, **_proj(d_in, d_out, lam, R))
    if kind == "train":
        n = logint(1, 32)
        hi = logint(8, max(8, min(2000, 40000000 // ((d_in + d_out) * n))))
        return dict(both, n=n, chunks=n, new_lo=max(1, hi // 4), new_hi=hi, count=logint(1, 24))
    if rng.random() < 0.6:
        most = max(1, int(2.5e8 // (R * (d_in + d_out) / lam)))      # adapters
        return dict(both, n=logint(1, 256), chunks=0, new_lo=1, new_hi=1, count=logint(1, min(128, most)))
    n = logint(1, 32)
    hi = logint(8, max(8, min(2000, 60000000 // ((d_in + d_out) * n))))
    return dict(both, n=n, chunks=rng.randint(1, n), new_lo=max(1, hi // 4), new_hi=hi, count=logint(1, 24))


# ---- what a case's batch looks like -----------------------------------------------------------------------

def batch(case):
    """(new tokens, adapter) of each request, and each adapter's rank."""
    r = random.Random(case["ragged"])
    lo, hi = case["new_lo"], case["new_hi"]
    fresh = [min(hi, int(lo * ((hi + 1) / lo) ** r.random())) if i < case["chunks"] else 1 for i in range(case["n"])]
    r.shuffle(fresh)
    deal = list(range(case["count"]))                                # every adapter occurs before one occurs twice
    r.shuffle(deal)
    which = [-1 if r.random() < case["bare"] else deal[i % len(deal)] for i in range(case["n"])]
    if max(which) < 0:
        which[0] = 0
    r.shuffle(which)
    R = case.get("R", 8)
    ranks = [r.choice([R, max(8, R // 2), max(8, R // 4)]) if case.get("mixed") else R for _ in range(case["count"])]
    ranks[0] = R
    return fresh, which, ranks


def tile_room(tokens, count):
    return -(-tokens // TILE) + min(tokens, count)


def sizes(case):
    """Elements of each tensor of an optimizer's case."""
    r = random.Random(case["ragged"])
    if not case["layers"]:
        return [min(case["hi"], max(case["lo"], int(case["lo"] * (case["hi"] / case["lo"]) ** r.random()))) for _ in range(case["tensors"])]
    h, f, R = {65: (8192, 22016, 256), 13: (5120, 13824, 128)}.get(case["ragged"], (4096, 11008, 128))
    one = [(i // 2) * R for o, i in ((h, h),) * 4 + ((f, h),) * 2 + ((h, f),) for i in (i, o)]
    return one * case["layers"]


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + stream) & (2**63 - 1))


def _normal(seed, stream, shape, std=1.0, dtype=BF16):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda", dtype=dtype).mul_(std)


def _ints(values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _two_to(x, top):
    """The smallest power of two that brings |x| within `top` = 1.75 * 2^k, and at least 2^-126."""
    mantissa, e = torch.frexp(x)                                     # x = mantissa * 2^e, 0.5 <= mantissa < 1
    k = math.frexp(top)[1]
    e = torch.where(mantissa <= 0.875, e - k, e - k + 1)
    return torch.where(x > 0, torch.ldexp(torch.ones_like(x), e.clamp(min=-126)), torch.full_like(x, 2.0 ** -126))


def prepare(case, seed):
    kind = case["kind"]
    st = {"kind": kind}
    if kind == "adamw":
        return _prepare_adamw(case, seed, st)
    fresh, which, ranks = batch(case)
    if kind == "groups":                                             # the same requests in another order, with other adapters
        both = [(m, a if a < 0 else (a + seed) % case["count"]) for m, a in zip(fresh, which)]
        random.Random(seed).shuffle(both)
        fresh, which = [m for m, _ in both], [a for _, a in both]
    starts = [0]
    for m in fresh:
        starts.append(starts[-1] + m)
    T = starts[-1]
    st["starts"], st["which"], st["count"] = _ints(starts), _ints(which), case["count"]
    if kind == "groups":
        st["tokens"] = -(-T // 64) * 64                              # a batch is padded to whole tiles
        return st
    # the groups of the step, which all projections share
    st["groups"] = _plain_groups(st["starts"], st["which"], case["count"], T)
    lengths = [0] * case["count"]
    for a, m in zip(which, fresh):
        if a >= 0:
            lengths[a] += m
    st["most"] = max(1, max(lengths))
    d_in, d_out, lam1, lam2 = (case[k] for k in ("d_in", "d_out", "lam1", "lam2"))
    st["lam1"], st["lam2"], st["R"] = lam1, lam2, case["R"]
    a_flat = torch.rand(sum(ranks) * (d_in // lam1), generator=_gen(seed, 1), device="cuda").mul_(2).sub_(1)
    a_flat = a_flat.mul_((lam1 / d_in) ** 0.5).to(BF16)
    b_flat = _normal(seed, 2, (sum(ranks) * (d_out // lam2),), 0.05)
    st["A"] = [x.view(-1, r) for x, r in zip(a_flat.split([r * (d_in // lam1) for r in ranks]), ranks)]
    st["B"] = [x.view(r, -1) for x, r in zip(b_flat.split([r * (d_out // lam2) for r in ranks]), ranks)]
    st["s"] = [(0.5, 1.0, 2.0)[a % 3] for a in range(case["count"])]
    st["X"], st["Y"] = _normal(seed, 3, (T, d_in)), _normal(seed, 4, (T, d_out))
    if kind == "train":
        st["dY"], st["dX"] = _normal(seed, 5, (T, d_out), 0.1), _normal(seed, 6, (T, d_in), 0.1)
        st["dA"] = [torch.empty(x.shape, dtype=F32, device="cuda") for x in st["A"]]
        st["dB"] = [torch.empty(x.shape, dtype=F32, device="cuda") for x in st["B"]]
    if own:                                                          # the handle of the loaded adapters
        from paper_2407_17029_amd import binding as qb
        ads = [qb.Adapter(A, B, lam1, lam2, s) for A, B, s in zip(st["A"], st["B"], st["s"])]
        st["table"] = qb.qblora_adapter_table(ads, d_in, d_out, R=case["R"],
                                              grads=list(zip(st["dA"], st["dB"])) if kind == "train" else None)
    return st


def _prepare_adamw(case, seed, st):
    n = sizes(case)
    room = [-(-k // 256) * 256 for k in n]
    at = [0]
    for k in room:
        at.append(at[-1] + k)
    total = at[-1]
    st["n"], st["room"], st["bits"], st["step"], st["clip"] = n, room, case["bits"], 100, 0.3 if case["clip"] else None
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, k in zip(at, n):
        inside[a:a + k] = True
    # gradients of very different sizes from tensor to tensor and from block to block, some of them zero
    size = torch.exp(_normal(seed, 1, (total // 256, 1), 1.5, F32)).mul_(1e-3)
    rows = lambda stream, std=1.0: _normal(seed, stream, (total // 256, 256), std, F32)  # noqa: E731
    seen = (inside & (torch.rand(total, generator=_gen(seed, 2), device="cuda") > 0.02)).view(-1, 256)
    st["g"] = (rows(3) * size * seen).view(-1)
    m = rows(4, 0.3) * size * seen
    v = rows(5).square_().add_(0.05).mul_(size * size * seen)
    w = rows(6, 0.02).view(-1) * inside
    st["p"] = w.to(BF16)
    st["w"] = w if case["master"] else None
    if case["bits"] == 8:
        st["ms"], st["vs"] = _two_to(m.abs().amax(1), 448.0), _two_to(v.amax(1), 57344.0)
        st["m"] = (m / st["ms"][:, None]).to(torch.float8_e4m3fn).view(-1)
        st["v"] = (v / st["vs"][:, None]).to(torch.float8_e5m2).view(-1)
    else:
        st["m"], st["v"] = m.view(-1), v.view(-1)
    st["rate"] = [(1.0, 4.0)[i % 2] for i in range(len(n))]          # A and B at rates of their own
    st["decay"] = [(0.01, 0.0)[i % 2] for i in range(len(n))]
    if own:                                                          # the handle of the tensors
        from paper_2407_17029_amd import binding as qb
        cut = lambda t: [x[:k] for x, k in zip(t.split(room), n)]  # noqa: E731
        blocks = lambda t: list(t.split([k // 256 for k in room]))  # noqa: E731
        st["list"] = qb.qblora_adamw_list(cut(st["p"]), cut(st["g"]), cut(st["m"]), cut(st["v"]),
                                          master=cut(st["w"]) if st["w"] is not None else None,
                                          m_scale=blocks(st["ms"]) if case["bits"] == 8 else None,
                                          v_scale=blocks(st["vs"]) if case["bits"] == 8 else None,
                                          rate=st["rate"], decay=st["decay"])
    return st


RATE, BETA1, BETA2, TINY, SEED = 1e-4, 0.9, 0.999, 1e-8, 12345


# ---- the operators in plain form ------------------------------------------------------------------------

def _plain_groups(starts, which, count, tokens):
    n = which.numel()
    t = torch.arange(tokens, device=which.device)
    request = torch.searchsorted(starts[1:].contiguous(), t.to(I32), right=True).clamp(max=n - 1)
    a = torch.where(t < starts[-1], which[request], -1)
    key, order = torch.sort(torch.where((a >= 0) & (a < count), a, count), stable=True)
    order = torch.where(key < count, order, -1)
    first = torch.searchsorted(key, torch.arange(count + 1, device=key.device, dtype=key.dtype))
    length = first[1:] - first[:-1]
    ends = torch.cumsum((length + TILE - 1) // TILE, 0)
    i = torch.arange(tile_room(tokens, count), device=key.device)
    of = torch.searchsorted(ends, i, right=True)
    real = of < count
    of = of.clamp(max=count - 1)
    nth = i - (ends - (length + TILE - 1) // TILE)[of]
    begin = first[of] + TILE * nth
    tiles = torch.stack([of, begin, (first[of + 1] - begin).clamp(max=TILE), torch.zeros_like(of)], 1)
    return {"first": first.to(I32), "order": order.to(I32), "tiles": torch.where(real[:, None], tiles, 0).to(I32)}


def _stacked(matrices, shape):
    """One fp32 array of all adapters' matrices, ranks filled up with zeros."""
    return torch.stack([torch.nn.functional.pad(x.to(F32), (0, shape[1] - x.shape[1], 0, shape[0] - x.shape[0])) for x in matrices])


def _rows(st):
    """Token of place l of each adapter, and whether there is one; [adapters, most]."""
    first, order = st["groups"]["first"].long(), st["groups"]["order"].long()
    place = first[:-1, None] + torch.arange(st["most"], device=first.device)[None, :]
    real = place < first[1:, None]
    return order[place.clamp(max=order.numel() - 1)].clamp(min=0), real


def _pooled(x, token, real, lam):
    rows = x.to(F32)[token] * real[:, :, None]
    return rows.view(*rows.shape[:2], -1, lam).sum(-1)


def _add(y, token, real, values):
    """y[token] += values where real, one rounding; the other rows stay."""
    T = y.shape[0]
    place = torch.full((T + 1,), -1, dtype=torch.int64, device=y.device)
    place.scatter_(0, torch.where(real, token, T).view(-1), torch.arange(real.numel(), device=y.device))
    more = values.reshape(real.numel(), -1)[place[:T].clamp(min=0)]
    y.copy_(torch.where(place[:T, None] >= 0, y.to(F32) + more, y.to(F32)))


def _plain_fwd(st):
    token, real = _rows(st)
    A = _stacked(st["A"], (st["A"][0].shape[0], st["R"]))
    B = _stacked(st["B"], (st["R"], st["B"][0].shape[1]))
    s = torch.tensor(st["s"], dtype=F32, device="cuda")[:, None, None]
    P = _pooled(st["X"], token, real, st["lam1"]) / st["lam1"]
    U = torch.bmm(P, A)
    _add(st["Y"], token, real, (s * torch.bmm(U, B)).repeat_interleave(st["lam2"], -1))
    return token, real, A, B, s, P, U


def _plain_train(st):
    token, real, A, B, s, P, U = _plain_fwd(st)
    dV = s * _pooled(st["dY"], token, real, st["lam2"])
    dU = torch.bmm(dV, B.transpose(1, 2).contiguous())
    dA, dB = torch.bmm(P.transpose(1, 2).contiguous(), dU), torch.bmm(U.transpose(1, 2).contiguous(), dV)
    dP = torch.bmm(dU, A.transpose(1, 2).contiguous()) / st["lam1"]
    _add(st["dX"], token, real, dP.repeat_interleave(st["lam1"], -1))
    for a, (x, y) in enumerate(zip(st["dA"], st["dB"])):
        x.copy_(dA[a, :, :x.shape[1]])
        y.copy_(dB[a, :y.shape[0]])
    return {"Y": st["Y"], "dX": st["dX"], "dA": st["dA"], "dB": st["dB"]}


def _wrap(x):
    return x & 0xffffffff


def _random(n, room, step):
    """32 random bits for every element, from its place in its tensor, the tensor's number, the step and the seed."""
    number = torch.repeat_interleave(torch.arange(len(n), device="cuda"), _ints(room, torch.int64), output_size=sum(room))
    start = torch.cumsum(_ints(room, torch.int64), 0) - _ints(room, torch.int64)
    e = torch.arange(sum(room), device="cuda") - start[number]
    key = (SEED * 0x85157AF5 + step * 0xD168AAAD) & 0xffffffff
    x = _wrap(e * 0x9E3779B1 + number * 0x632BE5AB + key)
    x = _wrap((x ^ (x >> 16)) * 0x6C8E9CF5)
    x = _wrap((x ^ (x >> 15)) * 0xB5297A4D)
    return x ^ (x >> 16)


def _to_8_bits(x, top, random16, drop, low, never_zero):
    """(values in units of the block's scale, scales): x rounded to one of its two neighbours with 23 - drop mantissa bits (equally
    spaced ones below `low`), the upper one the more often the nearer it is."""
    x = x.view(-1, 256)
    scale = _two_to(x.abs().amax(1), top)
    a = (x.abs() / scale[:, None]).view(-1)
    bits = a.view(I32).long() + (random16 << (drop - 16)) + (1 << (drop - 17))
    up = (bits >> drop << drop).to(I32).view(F32)
    step = 2.0 ** (23 - drop) / low
    q = torch.floor(a * step + (random16.to(F32) + 0.5) * 2.0 ** -16)
    if never_zero:
        q = torch.where(a > 0, q.clamp(min=1.0), 0.0)
    return torch.where(a >= low, up, q / step).copysign_(x.reshape(-1)), scale


def _plain_adamw(st):
    g, out = st["g"], {}
    if st["clip"] is not None:
        norm = g.to(F64).square().sum().sqrt()
        factor = (st["clip"] / (norm + 1e-6)).clamp(max=1.0).to(F32)
        out["norm"] = norm.to(F32)
        g = g * factor
    st["step"] += 1
    c1, c2 = 1.0 - BETA1 ** st["step"], 1.0 - BETA2 ** st["step"]
    room = _ints(st["room"], torch.int64)
    each = lambda v: torch.repeat_interleave(torch.tensor(v, dtype=F32, device="cuda"), room, output_size=g.numel())  # noqa: E731
    m, v = st["m"].to(F32), st["v"].to(F32)
    if st["bits"] == 8:
        m, v = (m.view(-1, 256) * st["ms"][:, None]).view(-1), (v.view(-1, 256) * st["vs"][:, None]).view(-1)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = (v * BETA2 + (g * g) * (1.0 - BETA2)).clamp(max=torch.finfo(F32).max)
    w = st["w"] if st["w"] is not None else st["p"].to(F32)
    rate = each([RATE * r for r in st["rate"]])
    w = w * (1.0 - rate * each(st["decay"])) - rate / c1 * (m / (torch.sqrt(v) / math.sqrt(c2) + TINY))
    random32 = _random(st["n"], st["room"], st["step"]) if st["bits"] == 8 or st["w"] is None else None
    if st["w"] is not None:
        st["w"].copy_(w)
        st["p"].copy_(w)
        out["w"] = st["w"]
    else:                                                            # to one of the two nearest, the nearer the more often
        random16 = _wrap(random32 * 0x9E3779B1) >> 16
        st["p"].copy_(((w.view(I32).long() + random16) >> 16 << 16).to(I32).view(F32))
    out["p"] = st["p"]
    if st["bits"] == 8:
        m, ms = _to_8_bits(m, 448.0, random32 & 0xffff, 20, 2.0 ** -6, False)
        v, vs = _to_8_bits(v, 57344.0, random32 >> 16, 21, 2.0 ** -14, True)
        st["ms"].copy_(ms)
        st["vs"].copy_(vs)
        out["ms"], out["vs"] = st["ms"], st["vs"]
    st["m"].copy_(m)
    st["v"].copy_(v)
    return {**out, "m": st["m"], "v": st["v"]}


def run(state):
    st, kind = state, state["kind"]
    if not own:
        if kind == "groups":
            return _plain_groups(st["starts"], st["which"], st["count"], st["tokens"])
        if kind == "serve":
            _plain_fwd(st)
            return st["Y"]
        return _plain_train(st) if kind == "train" else _plain_adamw(st)
    from paper_2407_17029_amd import binding as qb
    if kind == "groups":
        first, order, tiles = qb.qblora_adapter_groups(st["starts"], st["which"], st["count"], st["tokens"])
        return {"first": first, "order": order, "tiles": tiles}
    if kind == "adamw":
        out, clipped = {}, None
        if st["clip"] is not None:
            clipped = qb.qblora_grad_norm(st["list"], st["clip"])
            out["norm"] = clipped[0]
        st["step"] += 1
        qb.qblora_adamw_step(st["list"], st["step"], RATE, BETA1, BETA2, TINY, clip=clipped, seed=SEED)
        out.update({k: st[k] for k in ("p", "m", "v")})
        out.update({k: st[k] for k in ("ms", "vs") if st["bits"] == 8})
        return out if st["w"] is None else {**out, "w": st["w"]}
    groups = (st["groups"]["first"], st["groups"]["order"], st["groups"]["tiles"])
    if kind == "serve":
        return qb.qblora_adapters_fwd(st["table"], groups, st["X"], st["Y"])
    saved = torch.empty(qb.qblora_adapters_saved_bytes(st["table"], len(st["X"])), dtype=torch.uint8, device="cuda")
    qb.qblora_adapters_fwd(st["table"], groups, st["X"], st["Y"], saved=saved)
    qb.qblora_adapters_bwd(st["table"], groups, st["X"], st["dY"], dX=st["dX"], saved=saved)
    return {"Y": st["Y"], "dX": st["dX"], "dA": st["dA"], "dB": st["dB"]}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------------

def _exact_adapters(case, st):
    """Adapter by adapter, with the matrices that a merge would add to the weight applied as two products."""
    fresh, which, _ = batch(case)
    owner = torch.cat([torch.full((m,), a) for a, m in zip(which, fresh)]).cuda()
    lam1, lam2 = case["lam1"], case["lam2"]
    Y = st["Y"].to(F64)
    grads = {"dX": st["dX"].to(F64), "dA": [], "dB": []} if case["kind"] == "train" else {}
    for a, (A, B, s) in enumerate(zip(st["A"], st["B"], st["s"])):
        t = (owner == a).nonzero().view(-1)
        A, B = A.to(F64), B.to(F64)
        big = A.repeat_interleave(lam1, 0) / lam1                    # [d_in, R]
        x = st["X"][t].to(F64)
        Y[t] += s * (x @ big @ B).repeat_interleave(lam2, 1)
        if grads:
            dy = st["dY"][t].to(F64)
            dv = s * torch.stack([dy[:, i::lam2] for i in range(lam2)]).sum(0)
            du = dv @ B.t()
            grads["dB"].append((x @ big).t() @ dv)
            g = x.t() @ du / lam1
            grads["dA"].append(torch.stack([g[i::lam1] for i in range(lam1)]).sum(0))
            grads["dX"][t] += du @ big.t()
    return {"Y": Y, **grads} if grads else Y


def _exact_adamw(st):
    g, out = st["g"].to(F64), {}
    room = _ints(st["room"], torch.int64)
    each = lambda v: torch.tensor(v, dtype=F64, device="cuda").repeat_interleave(room)  # noqa: E731
    if st["clip"] is not None:
        out["norm"] = torch.linalg.vector_norm(g)
        g = g * min(1.0, st["clip"] / (float(out["norm"]) + 1e-6))
    t = st["step"] + 1
    m, v = st["m"].to(F64), st["v"].to(F64)
    if st["bits"] == 8:
        m, v = m * st["ms"].to(F64).repeat_interleave(256), v * st["vs"].to(F64).repeat_interleave(256)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    w = (st["w"] if st["w"] is not None else st["p"]).to(F64)
    lr = RATE * each(st["rate"])
    w = w - lr * (each(st["decay"]) * w + m / (1.0 - BETA1 ** t) / ((v / (1.0 - BETA2 ** t)).sqrt() + TINY))
    out["p"] = w if st["w"] is not None else None                    # without the master copy: a matter of the random bits
    if st["w"] is not None:
        out["w"] = w
    if st["bits"] == 8:                                              # so are the moments in 8 bits
        return {**out, "m": None, "v": None, "ms": None, "vs": None}
    return {**out, "m": m, "v": v}


def exact(case, seed):
    if case["kind"] == "groups":
        return None                                                  # whole numbers
    st = prepare(case, seed)
    return _exact_adamw(st) if case["kind"] == "adamw" else _exact_adapters(case, st)


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    if case["kind"] == "adamw":
        n = sum(sizes(case))
        states = 16 if case["bits"] == 32 else 4 + 16 / 256          # both moments, in and out
        weights = 4 + 4 + 2 if case["master"] else 2 + 2
        return {"bytes": n * (4 + states + weights), "flops": 12 * n}
    fresh, which, ranks = batch(case)
    T = sum(fresh)
    if case["kind"] == "groups":
        room = -(-T // 64) * 64
        return {"bytes": 8 * case["n"] + 4 + 4 * (case["count"] + 1) + 4 * room + 16 * tile_room(room, case["count"]), "flops": T}
    length = [0] * case["count"]
    for a, m in zip(which, fresh):
        if a >= 0:
            length[a] += m
    d_in, d_out = case["d_in"], case["d_out"]
    per = d_in // case["lam1"] + d_out // case["lam2"]               # elements of A and B for each of the rank's columns
    used = sum(length)
    weights = 2 * sum(r * per for r, m in zip(ranks, length) if m)
    product = 2 * sum(m * r * per for r, m in zip(ranks, length))
    if case["kind"] == "serve":
        return {"bytes": used * (2 * d_in + 4 * d_out) + weights, "flops": product}
    return {"bytes": used * (2 * d_in + 4 * d_out) + used * (2 * d_out + 4 * d_in) + weights + 4 * sum(ranks) * per,
            "flops": 3 * product}
