"""Which form a call on many adapters takes, batches that reach each of them, and batches whose results are exact.

The forms of the outputs' half: "few" (k_spread_few: tiles of up to 4 tokens in the vector ALU, longer ones 16 tokens at a time through
the matrix pipe), "slices" (k_spread, which adds up the rank sums' slices itself) and "parts" (k_spread on sums that were added up
and cut into bf16 parts in front of it)."""
import ctypes as C

import numpy as np

import adapters_util as au


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


# ---- results that are exact ------------------------------------------------------------------------------------

def parts(v, n):
    """v in n bf16 parts: the nearest bf16 value, that of what is left, and so on; their sum."""
    total = np.zeros_like(v)
    for _ in range(n):
        total = total + au.bf16(v - total)
    return total


class Cancelling(au.Batch):
    """Every token's term is m times powers of two, computed as (h + m) - h with |m| < 2^-8 h: nothing is left of it without the low
    part of the narrow factor, with it everything is exact.  forward: U has h + m and h, B opposite rows; else dU and the transpose of A.

    h = 1 + 2^-7 .. 2 with 8 significant bits, m = 65 .. 127 times 2^-15: the sum has 16, its nearest bf16 value is h, the rest m."""

    def __init__(self, seed, d_in, d_out, lam1, lam2, ranks, lengths, which, forward):
        super().__init__(seed, d_in, d_out, lam1, lam2, ranks, lengths, which)
        r = np.random.Generator(np.random.Philox(key=[seed, 13]))
        T, K, J = self.T, d_in // lam1, d_out // lam2
        self.s = [(1.0, 2.0)[a % 2] for a in range(self.count)]
        self.h, self.m = 1.0 + r.integers(1, 128, T) / 128.0, r.integers(65, 128, T) * r.choice([-1.0, 1.0], T) * 2.0 ** -15
        self.X, self.dY = np.zeros((T, d_in)), np.zeros((T, d_out))
        self.Y, self.dX = np.zeros((T, d_out)), np.zeros((T, d_in))
        wide = self.X if forward else self.dY
        n_wide, n_out, lam = (K, J, lam1) if forward else (J, K, lam2)
        self.want = np.zeros((T, n_out))                         # of every token, before the repetition
        self.sign = r.choice([-2.0, -1.0, 0.5, 1.0], n_out)
        for a, R in enumerate(ranks):
            if not R:
                continue
            f1, f2 = r.choice(n_wide, 2, replace=False)
            r1, r2 = r.choice(R, 2, replace=False)
            first, second = np.zeros((n_wide, R)), np.zeros((R, n_out))      # the two matrices, as forward takes them
            first[f1, r1] = first[f2, r1] = first[f1, r2] = 1.0
            second[r1], second[r2] = self.sign, -self.sign
            self.A[a], self.B[a] = (first, second) if forward else (second.T.copy(), first.T.copy())
            for t in np.flatnonzero(self.owner == a):
                # a mean of lam1 equal inputs; a sum of lam2 outputs of which one counts
                for f, value in ((f1, self.h[t]), (f2, self.m[t])):
                    if forward:
                        wide[t, f * lam:(f + 1) * lam] = value
                    else:
                        wide[t, f * lam + int(r.integers(lam))] = value
                self.want[t] = self.s[a] * self.m[t] * self.sign / (1.0 if forward else lam1)
        self.want = np.repeat(self.want, lam2 if forward else lam1, 1)


class LongNumbers(au.Batch):
    """One token counts, and each r of U and of dU is a number of 24 bits, made of three bf16 ones without rounding: its dA and dB are
    those numbers, or 0.  What two bf16 parts leave of each is more than 2^-20 of it."""

    def __init__(self, seed, d_in, d_out, lam1, lam2, R, T, token):
        super().__init__(seed, d_in, d_out, lam1, lam2, [R], [T], [0])
        r = np.random.Generator(np.random.Philox(key=[seed, 17]))
        K, J = d_in // lam1, d_out // lam2
        self.s = [2.0]
        self.X, self.dY = np.zeros((T, d_in)), np.zeros((T, d_out))
        ks, js = r.choice(K, 3, replace=False), r.choice(J, 3, replace=False)
        self.u, self.du = self._numbers(r, R), self._numbers(r, R)
        self.A[0], self.B[0] = np.zeros((K, R)), np.zeros((R, J))
        for k, j, u, du in zip(ks, js, self._fields(self.u), self._fields(self.du)):
            self.A[0][k], self.B[0][:, j] = u, du
            self.X[token, k * lam1:(k + 1) * lam1] = 1.0
            self.dY[token, j * lam2 + int(r.integers(lam2))] = 1.0
        self.dA, self.dB = np.zeros((K, R)), np.zeros((R, J))
        self.dA[ks], self.dB[:, js] = self.s[0] * self.du, self.s[0] * self.u[:, None]

    @staticmethod
    def _numbers(r, n):
        """1 .. 1.9, multiples of 2^-23, of which two parts leave more than 2^-19."""
        out = np.zeros(0)
        while len(out) < n:
            v = r.integers(1 << 23, int(1.9 * (1 << 23)), 8 * n) / float(1 << 23)
            out = np.concatenate([out, v[np.abs(v - parts(v, 2)) > 2.0 ** -19]])
        return out[:n]

    @staticmethod
    def _fields(v):
        """Bits 1 to 8, 9 to 16 and 17 to 24 of each number, whose sums in any order are multiples of 2^-23 below 2: exact in fp32."""
        high = np.floor(v * 128.0) / 128.0
        mid = np.floor((v - high) * 32768.0) / 32768.0
        return high, mid, v - high - mid


# A long number's gradient: the fp32 sums that make the number add three values, those of the gradient three parts, and pooling up to
# eight equal ones in three additions; at most eight of them round, by 2^-24 each (none does on the way that the values are
# built for).  What two parts leave is 2^-20 at least.
LONG_TOLERANCE = 8 * 2.0 ** -24


def rms_limit(T, K):
    """Root mean square error of a gradient's elements, relative to their own, for random inputs: sums of T products of which each is added
    in three parts, so 3 T additions onto partial sums that grow with the root of their number, each off by 2^-24 of them at
    most: sqrt(1.5 T) 2^-24.  The narrow factor's own sums of K products: sqrt(K / 2) 2^-24.  Eight more for scales, slices and pooling."""
    return 2.0 ** -24 * (1.5 * T + 0.5 * K + 8.0) ** 0.5


def rms(got, want):
    return float(np.sqrt(((got - want) ** 2).mean() / (want ** 2).mean()))


# ranks, lengths, which, form without saved sums; d_in = 512, lambda1 = 2, d_out = 576, lambda2 = 2
CANCELLING = [([16, 64, 8, 64], [1, 2, 4, 3], [1, 0, 3, 2], "few"), ([128, 40], [5, 7], [0, 1], "few"), ([0, 256, 0, 0], [20], [1], "few"),
              ([64, 24], [64, 9], [0, 1], "slices"), ([8], [100], [0], "slices"), ([128, 72], [70, 30], [1, 0], "parts"),
              ([256, 200], [64, 33], [0, 1], "parts"), ([264], [17], [0], "parts"), ([512, 480], [3, 20], [1, 0], "parts")]
# d_in, d_out, lambda1, lambda2, R, tokens, the one that counts
LONG = [(64, 64, 1, 1, 8, 1, 0), (128, 192, 2, 2, 24, 5, 3), (256, 512, 4, 8, 128, 40, 33), (512, 256, 8, 4, 136, 70, 69),
        (320, 576, 2, 1, 264, 3, 0), (128, 128, 2, 2, 32, 1100, 700)]                # the last: sums in two slices
# tokens, d_in, d_out, lambda, R
RANDOM = [(64, 64, 64, 1, 64), (64, 128, 128, 2, 32), (200, 256, 128, 4, 136), (130, 512, 512, 8, 24)]
