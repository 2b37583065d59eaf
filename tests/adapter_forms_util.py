"""Which form a call on many adapters takes, and batches that reach each of them.

The forms of the outputs' half: "few" (k_spread_few: tiles of up to 4 tokens in the vector ALU, longer ones 16 tokens at a time through
the matrix pipe), "slices" (k_spread, which adds up the rank sums' slices itself) and "parts" (k_spread on sums that were added up
and cut into bf16 parts in front of it)."""
import ctypes as C


def form(L, count, T, R, kept=False):
    """Of a forward call, by the library's own rules; kept: s U is saved."""
    pay, few = L["_ZN6qblora14rank_parts_payEili"], L["_ZN6qblora18spread_few_appliesEil"]
    pay.argtypes, pay.restype = [C.c_int, C.c_int64, C.c_int], C.c_bool
    few.argtypes, few.restype = [C.c_int, C.c_int64], C.c_bool
    if kept or pay(count, T, R):
        return "parts"
    return "few" if few(count, T) else "slices"


def idle_between(tokens, ranks, count):
    """(ranks, lengths, which) of a table of `count` adapters, those with tokens spread over it; the others are idle, every fifth of
    them with matrices of its own, the rest without."""
    numbers = [i * count // len(tokens) for i in range(len(tokens))]
    assert len(set(numbers)) == len(tokens)
    all_ranks = [8 if i % 5 == 0 else 0 for i in range(count)]
    for a, R in zip(numbers, ranks):
        all_ranks[a] = R
    return all_ranks, tokens, numbers


# ---- batches of every form -----------------------------------------------------------------------------------

# Tiles of 1 to 4 tokens, of 5 to 16 in one pass, with a remainder of 1 to 4 behind passes of 16 (17, 18, 20, 36), with one that goes through
# the matrix pipe again (21, 40), whole tiles, and adapters with a second tile
TOKENS = [1, 2, 3, 4, 5, 15, 16, 17, 18, 20, 21, 36, 40, 63, 64, 67]


def some_ranks(R, n):
    """R and lower ones, of which some fall into another step of 32 r than R."""
    return [max(8, r // 8 * 8) for r in (([R, R // 2, R, R // 8] * n)[:n])]


# lambda2, R, d_out, tokens, loaded adapters, form; d_in = 256, lambda1 = 2
FORMS = [(lam2, R, d_out, TOKENS, 60, "few") for lam2 in (1, 2, 4, 8) for R in (8, 64, 128, 136, 256) for d_out in (832,)]
# enough outputs for pieces of 256 rows, the last of them not a whole one
FORMS += [(lam2, R, 2112 * lam2, TOKENS, 60, "few") for lam2 in (1, 2, 4, 8) for R in (24, 200)]
# up to three tokens in all, for which less LDS is asked for
FORMS += [(lam2, R, 576, tokens, 3, "few") for lam2 in (1, 4, 8) for R in (16, 104, 256) for tokens in ([1], [2], [1, 1, 1], [3])]
# one adapter among idle ones
FORMS += [(lam2, 128, 640, [n], -(-n // 8), "few") for lam2 in (1, 4, 8) for n in (17, 20, 36, 64, 67)]
# eight tokens for each adapter of the table, and one more
FORMS += [(lam2, R, 640, [20, 3, 9 + more], 4, form_) for lam2 in (1, 4, 8) for R in (64, 256)
          for more, form_ in ((0, "few"), (1, "slices" if R == 64 else "parts"))]
