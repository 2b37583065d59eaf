"""What chooses the form of a call on many adapters, without a GPU: the batches of test_gpu_adapter_forms.py take the form that they are there
for, so that a rule that changes does not leave a form without tests."""
import pytest

import adapter_forms_util as af


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
