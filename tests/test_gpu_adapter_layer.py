"""The operators on many adapters and the optimizer's step as a model uses them (examples/decoder_layer.py): requests with adapters of
their own through whole layers, and adapters trained side by side, against the same computed one adapter at a time with the
single-adapter calls."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decoder_layer_example", os.path.join(ROOT, "examples", "decoder_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def near(got, want, what, limit):
    """Root of the mean square error over that of the values."""
    g, w = got.double(), want.double()
    err = ((g - w).square().mean() / w.square().mean()).sqrt().item()
    assert err <= limit, f"{what}: {err:.2e}"


def test_requests_with_adapters(example):
    """Prompts and single tokens of a batch with adapters, against each request by itself through the projections with its adapter (the
    single-adapter forward).  Both round every projection's output and the residual stream to bf16 (2^-9 of a value at most each, about
    a dozen of them a layer) and take the adapter term apart from the base product: a few times 2^-9 of the result's size."""
    from paper_2407_17029_amd import binding as qb
    layers = [example.DecoderLayer(512, 4, 2, 1024, seed=i) for i in range(2)]
    for i, l in enumerate(layers):
        l.load(3, rank=8, seed=20 + i)
    r = torch.Generator("cuda").manual_seed(3)
    prompts = [torch.randn(n, 512, device="cuda", generator=r).to(torch.bfloat16) for n in (70, 1, 33, 130, 20)]
    which = torch.tensor([2, 0, -1, 1, 2], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        first, outs, _, _ = example.serve(layers, prompts, 3, 16, which)
        none, none_outs, _, _ = example.serve(layers, prompts, 3, 16, torch.full_like(which, -1))
        base, base_outs, _, _ = example.serve(layers, prompts, 3, 16)
    assert torch.equal(none, base) and all(torch.equal(x, y) for x, y in zip(none_outs, base_outs))

    class Alone:
        def __init__(self, projection, number):
            self.weight, self.table = projection.weight, projection.table
            self.adapter = projection.table.adapters[number] if number >= 0 else None

        def __call__(self, x, groups=None):
            return qb.qblora_linear_fwd(self.weight, self.adapter, x)

    at = 0
    for i, p in enumerate(prompts):
        alone = []
        for l in layers:
            c = object.__new__(example.DecoderLayer)
            c.__dict__.update(l.__dict__)
            for name in ("qkv", "out", "gate_up", "down"):
                setattr(c, name, Alone(getattr(l, name), int(which[i])))
            alone.append(c)
        with torch.no_grad():
            # the inputs of the single tokens are what the batch gave: errors do not add up over the steps
            fed = [first[at + len(p) - 1]] + [y[i] for y in outs[:-1]]
            ones = torch.ones(512, dtype=torch.bfloat16, device="cuda")
            steps = [qb.qblora_rms_norm_fwd(f[None].contiguous(), ones, example.EPS)[0] for f in fed]
            want, _, _, _ = example.serve(alone, [torch.cat([p, *steps])], 0, 16)
        near(first[at:at + len(p)], want[:len(p)], f"prompt {i}", 0.02)
        near(torch.stack([y[i] for y in outs]), want[len(p):], f"single tokens {i}", 0.02)
        if int(which[i]) >= 0:                               # the adapters count: without them the result is another
            assert (first[at:at + len(p)].float() - base[at:at + len(p)].float()).abs().max() > 0.1
        at += len(p)


def test_adapters_side_by_side(example):
    """Loss and gradients of three adapters in one step, against the single-adapter calls on each one's sequences: between the two
    lie the roundings of bf16 activations and gradients."""
    length, which, hidden = 96, [0, 2, 0, 1], 256
    layer = example.DecoderLayer(hidden, 4, 2, 2 * hidden, seed=5)
    tuner = example.Tuner(layer, which, 3, length, rank=8)
    r = torch.Generator("cuda").manual_seed(8)
    x, target = (torch.randn(len(which) * length, hidden, device="cuda", generator=r).to(torch.bfloat16) for _ in range(2))
    with torch.no_grad():
        loss, dx, dw, _ = tuner.step(x, target, len(which))
        total, dws = 0.0, torch.zeros_like(dw)
        for a in range(3):
            mine = [i for i, w in enumerate(which) if w == a]
            rows = torch.cat([torch.arange(i * length, (i + 1) * length) for i in mine]).cuda()
            single = example.Trainer(layer, rank=8)
            single.qkv, single.out = tuner.adapters["qkv"][a], tuner.adapters["out"][a]
            part = len(mine) / len(which)                    # a step's loss is over its own tokens
            loss_a, dx_a, dw_a, grads = single.step(x[rows].contiguous(), target[rows].contiguous(), len(mine))
            total += part * loss_a
            dws += part * dw_a
            near(dx[rows], part * dx_a.float(), f"dx of {a}", 0.01)
            for name, (_, dA, dB) in zip(("qkv", "out"), grads):
                near(tuner.grads[name][a][0], part * dA, f"dA of {name} {a}", 0.01)
                near(tuner.grads[name][a][1], part * dB, f"dB of {name} {a}", 0.01)
    assert abs(loss - total) <= 1e-3 * total
    near(dw, dws, "dw", 0.01)


def test_steps_of_adapters_side_by_side(example):
    """Every adapter with tokens is moved by a step, one without keeps its values (no decay, a gradient of zero), parameters are the
    rounded masters, and the norm is that of the gradients."""
    layer = example.DecoderLayer(256, 4, 2, 512, seed=6)
    tuner = example.Tuner(layer, [0, 2], 4, 64, rank=8)
    r = torch.Generator("cuda").manual_seed(9)
    x, target = (torch.randn(128, 256, device="cuda", generator=r).to(torch.bfloat16) for _ in range(2))
    before = {n: [(a.A.clone(), a.B.clone()) for a in ads] for n, ads in tuner.adapters.items()}
    with torch.no_grad():
        for _ in range(3):
            _, _, dw, _ = tuner.step(x, target, 2)
            clip = tuner.update(dw)
            norm = sum(float(g.double().square().sum()) for pairs in tuner.grads.values() for p in pairs for g in p) + float(dw.double().square().sum())
            assert abs(float(clip[0]) - norm ** 0.5) <= 1e-6 * norm ** 0.5
    for n, ads in tuner.adapters.items():
        for i, a in enumerate(ads):
            same = [torch.equal(a.A, before[n][i][0]), torch.equal(a.B, before[n][i][1])]
            assert same == ([False, False] if i in (0, 2) else [True, True]), (n, i)
    params, _, _, _, masters, _, _ = tuner.list.tensors
    assert all(torch.equal(p, w.to(torch.bfloat16)) for p, w in zip(params, masters))
    assert all(torch.isfinite(p.float()).all() for p in params)


def test_adapted_projection_is_the_single_adapter_one():
    """One adapter for all tokens: base call and adapter call against the fused single-adapter calls, forward and backward."""
    import adapters_util as au
    from paper_2407_17029_amd import binding as qb
    r = torch.Generator("cuda").manual_seed(11)
    T, d_in, d_out, R, lam = 300, 512, 768, 32, 2
    qw = qb.qblora_quantize_blockwise(torch.randn(d_out, d_in, device="cuda", generator=r) * 0.02, 64, qb.QUANT_MINMAX_INT4)
    A = (torch.randn(d_in // lam, R, device="cuda", generator=r) * 0.06).to(torch.bfloat16)
    B = (torch.randn(R, d_out // lam, device="cuda", generator=r) * 0.1).to(torch.bfloat16)
    ad = qb.Adapter(A, B, lam, lam, 2.0)
    grads = [(torch.empty(A.shape, device="cuda"), torch.empty(B.shape, device="cuda"))]
    table = qb.qblora_adapter_table([ad], d_in, d_out, grads=grads)
    groups = qb.qblora_adapter_groups(au.dev([0, T]), au.dev([0]), 1, T)
    X, dY = (torch.randn(T, d, device="cuda", generator=r).to(torch.bfloat16) for d in (d_in, d_out))
    Y = qb.qblora_adapters_fwd(table, groups, X, qb.qblora_linear_fwd(qw, None, X))
    dX, _, _ = qb.qblora_linear_bwd(qw, None, X, dY)
    qb.qblora_adapters_bwd(table, groups, X, dY, dX=dX)
    wX, wA, wB = qb.qblora_linear_bwd(qw, ad, X, dY)
    # one more rounding of the base product, 2^-9 of it at most, and two roundings of the sum
    near(Y, qb.qblora_linear_fwd(qw, ad, X), "Y", 3 * 2.0 ** -9)
    near(dX, wX, "dX", 3 * 2.0 ** -9)
    near(grads[0][0], wA, "dA", 2.0 ** -15)                  # the single-adapter call's narrow factors have 16 bits
    near(grads[0][1], wB, "dB", 2.0 ** -15)
