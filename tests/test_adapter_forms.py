"""What chooses the form of a call on many adapters, without a GPU: the batches of test_gpu_adapter_forms.py take the form that they are there
for, so that a rule that changes does not leave a form without tests.  And the batches that show what is lost with a part of the narrow
factors: the mistake is made here, in the plain form, which then fails the GPU tests' tolerances."""
import numpy as np
import pytest

import adapter_forms_util as af
import adapters_util as au


@pytest.mark.parametrize("lam2,R,d_out,tokens,count,form", af.FORMS)
def test_form_of_each_batch(rules, lam2, R, d_out, tokens, count, form):
    assert af.form(rules.L, count, sum(tokens), R) == form
    ranks, lengths, which = af.idle_between(tokens, af.some_ranks(R, len(tokens)), count)
    assert max(ranks) <= R and ranks[which[0]] == R and len(ranks) == count and lengths == tokens


def test_batches_reach_every_part_of_the_form_for_few_tokens():
    """Every repetition with tiles of one, two and more tokens in the vector ALU, the matrix pipe, second passes of both kinds."""
    for lam2 in (1, 2, 4, 8):
        for step in (64, 128, 256):                          # inner ranks that share a form of the kernel
            lengths = {n for l, R, _, tokens, _, f in af.FORMS if l == lam2 and f == "few" and step // 2 < max(R, 64) <= step for n in tokens}
            tiles = {min(64, n - at) for n in lengths for at in range(0, n, 64)}
            assert {1, 2, 3, 4, 16, 17, 20, 36, 64} <= tiles and {m % 16 for m in tiles if m > 16} >= {0, 1, 2, 4, 5}
        pieces = {d_out // lam2 > 256 * 8 for l, _, d_out, _, _, _ in af.FORMS if l == lam2}
        assert pieces == {False, True}


def test_rules_at_their_limits(rules):
    for count in (1, 4, 500):
        assert af.form(rules.L, count, min(8 * count, 1023), 64) == "few"
        assert af.form(rules.L, count, 8 * count + 1, 64) == ("slices" if 8 * count + 1 < 1024 else "parts")
        assert af.form(rules.L, count, 8 * count + 1, 72) == "parts"
        assert af.form(rules.L, count, 1, 256) == "few" and af.form(rules.L, count, 1, 264) == "parts"
        assert af.form(rules.L, count, 1024, 8) == "parts" and af.form(rules.L, count, 1, 8, kept=True) == "parts"


@pytest.mark.parametrize("forward", [True, False])
@pytest.mark.parametrize("ranks,lengths,which,form", af.CANCELLING)
def test_cancelling_terms_need_both_parts(rules, ranks, lengths, which, form, forward):
    """The plain form gives exactly what the batch was built for; so does the narrow factor in two bf16 parts, while one part leaves
    nothing of any token's term."""
    assert af.form(rules.L, len(ranks), sum(lengths), max(ranks)) == form
    b = af.Cancelling(len(lengths), 512, 576, 2, 2, ranks, lengths, which, forward)
    got = b.forward()[0] if forward else b.backward()[0]
    assert np.array_equal(got, b.want) and (b.want != 0).all()
    assert np.array_equal(af.parts(b.h + b.m, 2), b.h + b.m) and np.array_equal(af.parts(b.h + b.m, 1), b.h)
    for x in (b.X, b.dY, *b.A, *b.B, b.want):
        assert np.array_equal(au.bf16(x), x)


@pytest.mark.parametrize("case", af.LONG)
def test_long_numbers_need_three_parts(case):
    """Likewise; with the third part left out every element that is not zero is off by more than the tolerance of the GPU test."""
    b = af.LongNumbers(case[4], *case)
    _, dA, dB, _, _, _ = b.backward()
    assert np.array_equal(dA[0], b.dA) and np.array_equal(dB[0], b.dB)
    for x in (b.X, b.dY, b.A[0], b.B[0]):
        assert np.array_equal(au.bf16(x), x)
    for x in (b.u, b.du):
        assert np.array_equal(af.parts(x, 3), x)
        assert (np.abs(af.parts(x, 2) - x) > af.LONG_TOLERANCE * x).all()


@pytest.mark.parametrize("case", af.RANDOM)
def test_random_gradients_need_three_parts(case):
    """With two parts the gradients' error passes the limit of the GPU test, with three it is far below."""
    T, d_in, d_out, lam, R = case
    b = au.Batch(T + R, d_in, d_out, lam, lam, [R], [T], [0])
    P, dV = au.pool(b.X, lam) / lam, b.s[0] * au.pool(b.dY, lam)
    U, dU = P @ b.A[0], dV @ b.B[0].T
    for n, off in ((2, True), (3, False)):
        assert (af.rms(P.T @ af.parts(dU, n), P.T @ dU) > af.rms_limit(T, d_out)) == off
        assert (af.rms(af.parts(U, n).T @ dV, U.T @ dV) > af.rms_limit(T, d_in)) == off
