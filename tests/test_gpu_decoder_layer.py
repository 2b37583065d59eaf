"""The example's decoder layers (examples/decoder_layer.py) against 64 bits, every operator in its place.

The reference keeps 64 bits throughout, on the weights as they are rounded for the contraction.  The layer rounds its activations
to bf16 about ten times on the way to an output (norms, projections, rotary positions, attention, gate, stream), each 2^-9 of
the value at most and independent of the others: 10^0.5 * 2^-9 / 3^0.5 = 0.004 of the output's root mean square is
expected, and at most 0.02 is allowed for two layers; single elements at most 0.15 of it (five deviations of 0.02, and half a
step of an element five times the mean)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _dense(oracle, projection):
    w = projection.weight
    return oracle.dequantize(w.codes.cpu().numpy(), w.scales.cpu().numpy(), w.beta.cpu().numpy(), w.codebook, 64, 2)


def _norm(x, w):
    import decoder_util as du
    return du.norm(x, w, 1e-5)[0]


class Plain:
    """A layer on the whole sequence of one request."""

    def __init__(self, oracle, layer):
        import decoder_util as du
        self.W = {n: _dense(oracle, getattr(layer, n)) for n in ("qkv", "out", "gate_up", "down")}
        self.norms = [du.host(w) for w in layer.norms]
        self.layer = layer
        self.freq = (10000.0 ** (-2.0 * np.arange(layer.dim // 2) / layer.dim)).astype(np.float32)

    def __call__(self, x):
        import decoder_util as du
        l, T = self.layer, len(x)
        y = (_norm(x, self.norms[0]) @ self.W["qkv"].T).reshape(T, -1, l.dim)
        q, k, v = np.split(y, (l.heads, l.heads + l.kv_heads), axis=1)
        q, k = (du.rope(t, np.arange(T), self.freq, False, 1.0) for t in (q, k))
        a = np.zeros_like(q)
        for h in range(l.heads):
            s = q[:, h] @ k[:, h * l.kv_heads // l.heads].T * l.dim ** -0.5
            s[np.triu_indices(T, 1)] = -np.inf
            e = np.exp(s - s.max(1, keepdims=True))
            a[:, h] = e @ v[:, h * l.kv_heads // l.heads] / e.sum(1, keepdims=True)
        x = x + a.reshape(T, -1) @ self.W["out"].T
        gate, up = np.split(_norm(x, self.norms[1]) @ self.W["gate_up"].T, 2, axis=1)
        return x + (gate / (1.0 + np.exp(-gate)) * up) @ self.W["down"].T


def _near(got, want, what):
    rms = np.sqrt(np.mean(want * want))
    err = got - want
    assert np.sqrt(np.mean(err * err)) <= 0.02 * rms, f"{what}: {np.sqrt(np.mean(err * err)) / rms:.4f}"
    assert np.abs(err).max() <= 0.15 * rms, f"{what}: {np.abs(err).max() / rms:.4f}"


@pytest.mark.parametrize("hidden,heads,kv_heads,page,lengths", [
    (256, 4, 2, 16, [1, 40, 17]),                                      # 58 tokens: the small-batch projections
    (512, 4, 4, 64, [300, 5, 128, 63]),                                # 496 tokens: the contraction above 256
])
def test_prompts_and_single_tokens(oracle, example, hidden, heads, kv_heads, page, lengths):
    import decoder_util as du
    r = np.random.Generator(np.random.Philox(key=[hidden, 5]))
    layers = [example.DecoderLayer(hidden, heads, kv_heads, 2 * hidden, seed=i) for i in range(2)]
    plain = [Plain(oracle, l) for l in layers]
    prompts = [du.bf16(r.standard_normal((n, hidden))) for n in lengths]
    steps = 5
    with torch.no_grad():
        first, outs, _, _ = example.serve(layers, [du.dev_bf16(p) for p in prompts], steps, page)
    torch.cuda.synchronize()
    first, outs = du.host(first), [du.host(y) for y in outs]
    at = 0
    for i, p in enumerate(prompts):
        # the inputs of the single tokens are the outputs that the layers gave: errors do not add up over the steps
        fed = [first[at + len(p) - 1]] + [y[i] for y in outs[:-1]]
        x = np.concatenate([p, [du.bf16(_norm(f[None], 1.0)[0]) for f in fed]])
        for l in plain:
            x = l(x)
        _near(first[at:at + len(p)], x[:len(p)], f"prompt {i}")
        _near(np.array([y[i] for y in outs]), x[len(p):], f"single tokens {i}")
        at += len(p)


def test_training_step(example):
    """The gradients of the adapters, the norm's weight and the input against torch's own in fp32 through the dense layer
    (weights rebuilt by the contraction itself); descent lowers the loss."""
    import decoder_util as du
    from paper_2407_17029_amd import binding as qb
    hidden, sequences, length = 256, 2, 64
    layer = example.DecoderLayer(hidden, 4, 2, 2 * hidden, seed=3)
    trainer = example.Trainer(layer, rank=8)
    r = np.random.Generator(np.random.Philox(key=[9, 6]))
    x, target = (du.dev_bf16(r.standard_normal((sequences * length, hidden))) for _ in range(2))
    with torch.no_grad():
        loss, dx, dw, grads = trainer.step(x, target, sequences)
        dense = {n: qb.qblora_linear_fwd(getattr(layer, n).weight, None, torch.eye(hidden, dtype=torch.bfloat16, device="cuda")).float().t()
                 for n in ("qkv", "out")}
    leaves = {"x": x.float(), "w": trainer.norm.float()}
    for n, a in (("qkv", trainer.qkv), ("out", trainer.out)):
        leaves[n + "A"], leaves[n + "B"] = a.A.float(), a.B.float()
    leaves = {n: t.clone().requires_grad_() for n, t in leaves.items()}

    def adapted(h, name):
        lam = trainer.qkv.lambda1
        pooled = h.view(len(h), -1, lam).mean(2)
        return h @ dense[name].t() + (pooled @ leaves[name + "A"] @ leaves[name + "B"]).repeat_interleave(lam, 1)

    def rope(t):
        angle = torch.arange(length, device="cuda").repeat(sequences).double()[:, None] * trainer.freq.double()[None]
        c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
        a, b = t.chunk(2, 2)
        return torch.cat([a * c - b * s, b * c + a * s], 2)

    h = leaves["x"] * torch.rsqrt(leaves["x"].square().mean(1, keepdim=True) + 1e-5) * leaves["w"]
    q, k, v = layer.split(adapted(h, "qkv"))
    a = trainer.attention(rope(q), rope(k), v, sequences)
    diff = leaves["x"] + adapted(a, "out") - target.float()
    want = diff.square().sum() / (2 * len(x))
    want.backward()
    assert abs(loss - want.item()) <= 0.02 * want.item()
    got = {"x": dx, "w": dw, "qkvA": grads[0][1], "qkvB": grads[0][2], "outA": grads[1][1], "outB": grads[1][2]}
    for n, t in leaves.items():
        _near(du.host(got[n]), du.host(t.grad), n)
    with torch.no_grad():
        losses = example.train(trainer, x, target, sequences, 6, 0.02)
    assert losses[-1] < losses[0]
