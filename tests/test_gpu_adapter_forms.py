"""Every form of the outputs' half of the adapter terms on the GPU, in tables of which few adapters have tokens, against the plain form in 64
bits (tests/adapters_util.py).  test_adapter_forms.py asserts that the batches take the forms that they are meant for."""
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
