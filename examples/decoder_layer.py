#!/usr/bin/env python3
"""Decoder layers on 4-bit weights, served and trained with the library's operators.

serve()  a batch of requests of different lengths: their prompts in one call, then single tokens, every step of which is one
         replay of a HIP graph (the tables of pages, norms, projections, rotary positions into the cache, attention).
         With adapters loaded, every request has one of its own (or none) beside the shared projections.
train()  the attention half of a layer under balanced adapters, forward and backward, with the library's norms, projections
         and rotary positions; attention itself, which has no backward pass in the library, is torch's in fp32.
tune()   the same for several adapters side by side on one frozen layer, each on sequences of its own, stepped by AdamW with
         moments in 8 bits.

    python examples/decoder_layer.py [--hidden 4096 --heads 32 --kv-heads 8 --intermediate 11008 --layers 2
                                      --requests 16 --prompt 512 --new 64 --page 64 --adapters 4]

The weights are random.  Prints one line per phase."""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2407_17029_amd import binding as qb  # noqa: E402

BF16 = torch.bfloat16
EPS = 1e-5


class Projection:
    """A 4-bit weight: the small-batch kernels up to 256 tokens, the contraction of the fine-tuning path above."""

    def __init__(self, d_out, d_in, generator):
        W = torch.randn(d_out, d_in, device="cuda", generator=generator) * d_in ** -0.5
        self.weight = qb.qblora_quantize_blockwise(W, 64, qb.QUANT_MINMAX_INT4, tiled=False)
        self.pack = qb.qblora_decode_pack(self.weight)
        self.table = None

    def load(self, adapters):
        """Adapters by number, for batches that say which request has which."""
        self.table = qb.qblora_adapter_table(adapters, self.weight.d_in, self.weight.d_out)

    def __call__(self, x, groups=None):
        if x.shape[0] <= 256:
            y = qb.qblora_linear_decode(self.weight, x, pack=self.pack)
        else:
            y = qb.qblora_linear_fwd(self.weight, None, x)
        return y if groups is None or self.table is None else qb.qblora_adapters_fwd(self.table, groups, x, y)


class DecoderLayer:
    def __init__(self, hidden, heads, kv_heads, intermediate, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.hidden, self.heads, self.kv_heads, self.dim = hidden, heads, kv_heads, hidden // heads
        self.qkv = Projection((heads + 2 * kv_heads) * self.dim, hidden, g)
        self.out = Projection(hidden, hidden, g)
        self.gate_up = Projection(2 * intermediate, hidden, g)
        self.down = Projection(hidden, intermediate, g)
        self.norms = [(1.0 + 0.1 * torch.randn(hidden, device="cuda", generator=g)).to(BF16) for _ in range(2)]

    def split(self, y):
        """q, k, v of a joint projection, where they lie."""
        return y.view(len(y), -1, self.dim).split((self.heads, self.kv_heads, self.kv_heads), 1)

    def __call__(self, delta, stream, batch, cache, freq):
        """delta: what the layer before adds to the residual stream (the stream itself in front of the first layer, then
        stream is None)."""
        h, stream, _ = qb.qblora_rms_norm_fwd(delta, self.norms[0], EPS, residual=stream)
        q, k, v = self.split(self.qkv(h, batch.groups))
        q = qb.qblora_rope_cache(q, k, v, batch.positions, batch.slots, freq, *cache)
        a = qb.qblora_paged_attention(q, *cache, batch.table, batch.starts, batch.context, self.dim ** -0.5,
                                      max_new=batch.max_new)
        h, stream, _ = qb.qblora_rms_norm_fwd(self.out(a.view(len(a), -1), batch.groups), self.norms[1], EPS, residual=stream)
        gate, up = self.gate_up(h, batch.groups).chunk(2, 1)
        return self.down(torch.nn.functional.silu(gate) * up, batch.groups), stream

    def load(self, count, rank=16, lam=2, seed=2):
        """`count` random adapters on every projection, the ranks of every other one half as high."""
        g = torch.Generator("cuda").manual_seed(seed)
        for p in (self.qkv, self.out, self.gate_up, self.down):
            p.load([balanced_adapter(p, rank if i % 2 == 0 else rank // 2, lam, g) for i in range(count)])


def balanced_adapter(projection, rank, lam, generator):
    w, R = projection.weight, rank * lam
    A = (torch.randn(w.d_in // lam, R, device="cuda", generator=generator) * (w.d_in // lam) ** -0.5).to(BF16)
    B = (torch.randn(R, w.d_out // lam, device="cuda", generator=generator) * 0.02).to(BF16)
    return qb.Adapter(A, B, lam, lam, 1.0)


class Batch:
    """The requests of a server: block table and lengths on the device, advanced there.  which: the number of each request's
    adapter (-1: none) of `adapters` that are loaded."""

    def __init__(self, requests, longest, page, pages, which=None, adapters=0):
        self.page, self.which, self.adapters, self.groups = page, which, adapters, None
        self.table = torch.full((requests, -(-longest // page)), -1, dtype=torch.int32, device="cuda")
        self.context = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, device="cuda").to(torch.int32)
        self.order = torch.arange(pages, dtype=torch.int32, device="cuda")

    def begin(self, fresh, tokens, max_new):
        """Pages, positions and slots for `fresh` new tokens of each request, `tokens` of them together."""
        self.fresh, self.max_new = fresh, max_new
        self.starts, self.positions, self.slots, self.taken = qb.qblora_page_tables(self.context, fresh, self.page, self.free,
                                                                                    self.table, tokens)
        if self.which is not None:                                         # once for all projections of all layers
            self.groups = qb.qblora_adapter_groups(self.starts, self.which, self.adapters, tokens)

    def end(self):
        self.context += self.fresh
        pages = len(self.free)                                             # the list without its first `taken` entries
        moved = self.free[((self.order + self.taken) % pages).long()]
        self.free.copy_(torch.where(self.order < pages - self.taken, moved, -1))


def caches(layers, pages, page):
    """Keys and values of every layer; the layers share the block table."""
    return [(torch.zeros(pages, l.kv_heads, l.dim // 8, page, 8, dtype=BF16, device="cuda"),
             torch.zeros(pages, l.kv_heads, page // 8, l.dim, 8, dtype=BF16, device="cuda")) for l in layers]


def run(layers, x, batch, kv, freq):
    """x [tokens, hidden] through the layers; the residual stream behind the last."""
    delta, stream = x, None
    for layer, cache in zip(layers, kv):
        delta, stream = layer(delta, stream, batch, cache, freq)
    return stream + delta


def serve(layers, prompts, steps, page, which=None):
    """Prompts ([length, hidden] each) in one call, then `steps` single tokens of every request, whose inputs are the last
    outputs, normed.  which (int32 [requests]): each request's adapter, if the layers have some loaded.  Returns the outputs of
    the prompts, those of the steps, and the seconds of the prompts and of a step (0 without a second one: the first is not
    replayed)."""
    hidden = layers[0].hidden
    ones = torch.ones(hidden, dtype=BF16, device="cuda")
    lengths = [len(p) for p in prompts]
    pages = sum(-(-(n + steps) // page) for n in lengths)
    adapters = layers[0].qkv.table.count if which is not None else 0
    batch, kv = Batch(len(prompts), max(lengths) + steps, page, pages, which, adapters), caches(layers, pages, page)
    freq, _ = qb.qblora_rope_frequencies(layers[0].dim)
    fresh = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    x = torch.cat(prompts)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    batch.begin(fresh, len(x), max(lengths))
    first = run(layers, x, batch, kv, freq)
    last = batch.starts[1:].long() - 1
    batch.end()
    torch.cuda.synchronize()
    t1 = time.perf_counter()

    one = torch.ones_like(fresh)
    x, y = first[last], torch.empty(len(prompts), hidden, dtype=BF16, device="cuda")

    def step():
        batch.begin(one, len(prompts), 1)
        h, _, _ = qb.qblora_rms_norm_fwd(x, ones, EPS)
        y.copy_(run(layers, h, batch, kv, freq))
        batch.end()
        x.copy_(y)

    outs, seconds = [], 0.0
    if steps:
        step()                                                             # loads what must be there before a capture
        outs.append(y.clone())
    if steps > 1:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        torch.cuda.synchronize()
        t2 = time.perf_counter()
        for _ in range(steps - 1):
            graph.replay()
            outs.append(y.clone())
        torch.cuda.synchronize()
        seconds = (time.perf_counter() - t2) / (steps - 1)
    return first, outs, t1 - t0, seconds


class Trainer:
    """The attention half of a layer, out = x + Wo attention(rope(Wqkv norm(x))), on sequences of one length, with balanced
    adapters on both projections; everything but the adapters and the norm's weight is frozen."""

    def __init__(self, layer, rank=16, lam=2, seed=1):
        g = torch.Generator("cuda").manual_seed(seed)
        self.layer, self.norm = layer, layer.norms[0].clone()
        self.qkv, self.out = balanced_adapter(layer.qkv, rank, lam, g), balanced_adapter(layer.out, rank, lam, g)
        self.freq, _ = qb.qblora_rope_frequencies(layer.dim)

    def forward(self, name, x):
        return qb.qblora_linear_fwd(getattr(self.layer, name).weight, getattr(self, name), x)

    def backward(self, name, x, dy):
        return qb.qblora_linear_bwd(getattr(self.layer, name).weight, getattr(self, name), x, dy)

    def attention(self, q, k, v, sequences):
        """Causal attention in fp32 on [T, heads, dim], each sequence by itself."""
        q, k, v = (t.float().view(sequences, -1, t.shape[1], t.shape[2]).transpose(1, 2).contiguous() for t in (q, k, v))
        group = self.layer.heads // self.layer.kv_heads
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * self.layer.dim ** -0.5
        causal = torch.ones(scores.shape[-2:], dtype=torch.bool, device="cuda").tril()
        y = torch.matmul(scores.masked_fill(~causal, float("-inf")).softmax(-1), v)
        return y.transpose(1, 2).reshape(-1, self.layer.heads * self.layer.dim)

    def step(self, x, target, sequences):
        """Loss sum((out - target)^2) / 2 / T and its gradients: of x, the norm's weight and the adapters' A and B."""
        layer, T = self.layer, len(x)
        positions = torch.arange(T // sequences, dtype=torch.int32, device="cuda").repeat(sequences)
        h, _, rstd = qb.qblora_rms_norm_fwd(x, self.norm, EPS, keep=True)
        q, k, v = layer.split(self.forward("qkv", h))
        q, k = qb.qblora_rope_fwd(q, k, positions, self.freq)
        with torch.enable_grad():
            leaves = [t.detach().float().requires_grad_() for t in (q, k, v)]
            a = self.attention(*leaves, sequences)
        a16 = a.detach().to(BF16)
        y = self.forward("out", a16)
        diff = x.float() + y.float() - target.float()
        loss = float((diff * diff).sum()) / (2 * T)

        dout = (diff / T).to(BF16)
        da, dA_out, dB_out = self.backward("out", a16, dout)
        dq, dk, dv = (g.to(BF16).contiguous() for g in torch.autograd.grad(a, leaves, da.float()))
        joint = torch.empty(T, layer.qkv.weight.d_out, dtype=BF16, device="cuda")
        q_part, k_part, v_part = layer.split(joint)
        qb.qblora_rope_bwd(dq, dk, positions, self.freq, dq_out=q_part, dk_out=k_part)
        v_part.copy_(dv)
        dh, dA_qkv, dB_qkv = self.backward("qkv", h, joint)
        dx, dw = qb.qblora_rms_norm_bwd(x, self.norm, rstd, dh, dtotal=dout)
        return loss, dx, dw, [(self.qkv, dA_qkv, dB_qkv), (self.out, dA_out, dB_out)]


class Tuner(Trainer):
    """Several adapters side by side on one frozen layer: sequence i trains adapter which[i].  The base products and their
    gradients are one call for all of them, each adapter's term and gradients come from its own tokens, and one AdamW step
    moves all of them and the norm's weight."""

    def __init__(self, layer, which, count, length, rank=16, lam=2, seed=1, rate=1e-3, clip=1.0):
        super().__init__(layer, rank, lam, seed)
        g = torch.Generator("cuda").manual_seed(seed)
        starts = torch.arange(len(which) + 1, dtype=torch.int32, device="cuda") * length
        self.groups = qb.qblora_adapter_groups(starts, torch.tensor(which, dtype=torch.int32, device="cuda"), count, len(which) * length)
        self.rate, self.clip, self.step_number, self.saved = rate, clip, 0, {}
        self.adapters, self.grads, self.tables = {}, {}, {}
        for name in ("qkv", "out"):
            p = getattr(layer, name)
            self.adapters[name] = [balanced_adapter(p, rank, lam, g) for _ in range(count)]
            self.grads[name] = [(torch.zeros(a.A.shape, device="cuda"), torch.zeros(a.B.shape, device="cuda")) for a in self.adapters[name]]
            self.tables[name] = qb.qblora_adapter_table(self.adapters[name], p.weight.d_in, p.weight.d_out, grads=self.grads[name])
        self.dw = torch.zeros(layer.hidden, device="cuda")
        params = [m for ads in self.adapters.values() for a in ads for m in (a.A, a.B)] + [self.norm]
        grads = [g for pairs in self.grads.values() for pair in pairs for g in pair] + [self.dw]
        like = lambda dtype: [torch.zeros(t.shape, dtype=dtype, device="cuda") for t in params]  # noqa: E731
        scales = lambda: [torch.zeros(-(-t.numel() // 256), device="cuda") for t in params]  # noqa: E731
        self.list = qb.qblora_adamw_list(params, grads, like(torch.float8_e4m3fn), like(torch.float8_e5m2),
                                         master=[t.float() for t in params], m_scale=scales(), v_scale=scales())

    def forward(self, name, x):
        table = self.tables[name]
        saved = torch.empty(qb.qblora_adapters_saved_bytes(table, len(x)), dtype=torch.uint8, device="cuda")
        self.saved[name] = saved
        y = qb.qblora_linear_fwd(getattr(self.layer, name).weight, None, x)
        return qb.qblora_adapters_fwd(table, self.groups, x, y, saved=saved)

    def backward(self, name, x, dy):
        dx, _, _ = qb.qblora_linear_bwd(getattr(self.layer, name).weight, None, x, dy)
        qb.qblora_adapters_bwd(self.tables[name], self.groups, x, dy, dX=dx, saved=self.saved[name])
        return dx, None, None                                              # the adapters' gradients are in their places

    def update(self, dw):
        self.dw.copy_(dw)
        self.step_number += 1
        clip = qb.qblora_grad_norm(self.list, self.clip)
        qb.qblora_adamw_step(self.list, self.step_number, self.rate, clip=clip, seed=self.step_number)
        return clip


def tune(tuner, x, target, sequences, steps):
    """The losses of so many steps."""
    losses = []
    for _ in range(steps):
        loss, _, dw, _ = tuner.step(x, target, sequences)
        tuner.update(dw)
        losses.append(loss)
    return losses


def train(trainer, x, target, sequences, steps, rate):
    """Descent in which every matrix moves against its gradient by `rate` of its own size; the losses."""
    losses = []
    masters = [[t.float() for t in (a.A, a.B)] for a in (trainer.qkv, trainer.out)]
    for _ in range(steps):
        loss, _, _, grads = trainer.step(x, target, sequences)
        losses.append(loss)
        for (adapter, dA, dB), master in zip(grads, masters):
            for m, p, g in zip(master, (adapter.A, adapter.B), (dA, dB)):
                m -= g * (rate * m.norm() / g.norm().clamp_min(1e-30))
                p.copy_(m)
    return losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("intermediate", 11008), ("layers", 2), ("requests", 16),
                        ("prompt", 512), ("new", 64), ("page", 64), ("adapters", 4)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args(argv)
    layers = [DecoderLayer(a.hidden, a.heads, a.kv_heads, a.intermediate, seed=i) for i in range(a.layers)]
    g = torch.Generator("cuda").manual_seed(7)
    lengths = [max(1, a.prompt * (i + 1) // a.requests) for i in range(a.requests)]
    prompts = [torch.randn(n, a.hidden, device="cuda", generator=g).to(BF16) for n in lengths]
    with torch.no_grad():
        serve(layers, prompts, 3, a.page)                                  # loads kernels, fills the allocator
        _, _, first, rest = serve(layers, prompts, a.new, a.page)
    print(f"prompts: {sum(lengths)} tokens of {a.requests} requests in {1e3 * first:.2f} ms", flush=True)
    if a.new > 1:
        print(f"single tokens: {a.new - 1} steps of {a.requests} requests, {1e6 * rest:.0f} us each "
              f"({a.layers} layers)", flush=True)
    if a.adapters:
        for i, l in enumerate(layers):
            l.load(a.adapters, seed=100 + i)
        which = torch.arange(a.requests, dtype=torch.int32, device="cuda") % (a.adapters + 1) - 1
        with torch.no_grad():
            serve(layers, prompts, 3, a.page, which)
            _, _, first, rest = serve(layers, prompts, a.new, a.page, which)
        print(f"with {a.adapters} adapters: prompts {1e3 * first:.2f} ms, single tokens {1e6 * rest:.0f} us a step", flush=True)
    trainer = Trainer(layers[0])
    x = torch.randn(2 * 256, a.hidden, device="cuda", generator=g).to(BF16)
    target = x.roll(1, 0)
    with torch.no_grad():
        losses = train(trainer, x, target, 2, 5, 0.02)
    print("training: losses " + " ".join(f"{v:.3f}" for v in losses), flush=True)
    if a.adapters:
        tuner = Tuner(layers[0], [i % a.adapters for i in range(2 * a.adapters)], a.adapters, 256)
        x = torch.randn(2 * a.adapters * 256, a.hidden, device="cuda", generator=g).to(BF16)
        with torch.no_grad():
            losses = tune(tuner, x, x.roll(1, 0), 2 * a.adapters, 5)
        print(f"{a.adapters} adapters side by side: losses " + " ".join(f"{v:.3f}" for v in losses), flush=True)


if __name__ == "__main__":
    main()
