"""Every form of the outputs' half of the adapter terms on the GPU, in tables of which few adapters have tokens, against the plain form in 64
bits (tests/adapters_util.py), and batches whose results need every bf16 part of the narrow factors.  test_adapter_forms.py asserts
that the batches take the forms that they are meant for, and that they fail with a part left out."""
import numpy as np
import pytest
import torch

import adapter_forms_util as af
import adapters_util as au

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_amd import binding
    return binding


@pytest.mark.parametrize("lam2,R,d_out,tokens,count,form", af.FORMS)
def test_forward_of_each_form(qb, rules, lam2, R, d_out, tokens, count, form):
    """Each adapter's tokens against its own matrices, whole rows, with guards around the outputs and NaN in the workspace."""
    assert af.form(rules.L, count, sum(tokens), R) == form
    ranks, lengths, which = af.idle_between(tokens, af.some_ranks(R, len(tokens)), count)
    b = au.Batch(R + lam2, 256, d_out, 2, lam2, ranks, lengths, which)
    table, groups = b.table(qb, R=R), b.groups(qb)
    room = torch.full((b.T + 2, d_out), 3.0, dtype=torch.bfloat16, device=au.DEV)
    Y = room[1:1 + b.T]
    Y.copy_(au.dev_bf16(b.Y))
    ws = torch.full((qb.qblora_adapters_workspace_bytes(table, b.T) // 4,), float("nan"), device=au.DEV)
    qb.qblora_adapters_fwd(table, groups, au.dev_bf16(b.X), Y, workspace=ws)
    want, size = b.forward()
    au.assert_rows(Y, want, size, b.owner, b.Y, b.d_in, R, "Y")
    assert (room[0] == 3.0).all() and (room[-1] == 3.0).all()


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("ranks,lengths,which,form", af.CANCELLING)
def test_low_parts_reach_the_outputs(qb, ranks, lengths, which, form, kept):
    """Every sum and every result is exact, so that the outputs are equal to the plain form's."""
    b = af.Cancelling(len(lengths), 512, 576, 2, 2, ranks, lengths, which, True)
    table, groups, Y = b.table(qb), b.groups(qb), au.dev_bf16(b.Y)
    saved = torch.empty(qb.qblora_adapters_saved_bytes(table, b.T), dtype=torch.uint8, device=au.DEV) if kept else None
    qb.qblora_adapters_fwd(table, groups, au.dev_bf16(b.X), Y, saved=saved)
    assert np.array_equal(au.host(Y), b.want)


@pytest.mark.parametrize("gradients", [False, True])
@pytest.mark.parametrize("ranks,lengths,which,form", af.CANCELLING)
def test_low_parts_reach_the_inputs(qb, ranks, lengths, which, form, gradients):
    b = af.Cancelling(len(lengths), 512, 576, 2, 2, ranks, lengths, which, False)
    table, groups, dX = b.table(qb, grads=b.grads()), b.groups(qb), au.dev_bf16(b.dX)
    qb.qblora_adapters_bwd(table, groups, au.dev_bf16(b.X), au.dev_bf16(b.dY), dX=dX, gradients=gradients)
    assert np.array_equal(au.host(dX), b.want)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("case", af.LONG)
def test_gradients_hold_24_bits(qb, case, kept):
    b = af.LongNumbers(case[4], *case)
    grads = b.grads()
    table, groups, X = b.table(qb, grads=grads), b.groups(qb), au.dev_bf16(b.X)
    saved = None
    if kept:
        saved = torch.empty(qb.qblora_adapters_saved_bytes(table, b.T), dtype=torch.uint8, device=au.DEV)
        qb.qblora_adapters_fwd(table, groups, X, au.dev_bf16(b.Y), saved=saved)
    qb.qblora_adapters_bwd(table, groups, X, au.dev_bf16(b.dY), saved=saved)
    for name, got, want in (("dA", grads[0][0], b.dA), ("dB", grads[0][1], b.dB)):
        err = np.abs(got.cpu().numpy().astype(np.float64) - want)
        assert (err <= af.LONG_TOLERANCE * np.abs(want)).all(), f"{name}: {(err / np.where(want == 0, 1.0, want)).max():.3e}"


@pytest.mark.parametrize("case", af.RANDOM)
def test_gradients_are_as_close_as_fp32_products(qb, case):
    T, d_in, d_out, lam, R = case
    b = au.Batch(T + R, d_in, d_out, lam, lam, [R], [T], [0])
    grads = b.grads()
    qb.qblora_adapters_bwd(b.table(qb, grads=grads), b.groups(qb), au.dev_bf16(b.X), au.dev_bf16(b.dY))
    _, dA, dB, _, _, _ = b.backward()
    for name, got, want, K in (("dA", grads[0][0], dA[0], d_out), ("dB", grads[0][1], dB[0], d_in)):
        off = af.rms(got.cpu().numpy().astype(np.float64), want)
        assert off <= af.rms_limit(T, K), f"{name}: {off:.3e}"
