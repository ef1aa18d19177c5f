"""Attention over two keys in fp32 whose operands need all three of their bf16 terms, with bounds that a lost term or product
passes: inputs, bounds, and a model of the products in terms.

An operand +-(1 + a 2^-8 + b 2^-16), a and b of 0 or 1, b only where a is, is the terms 1, a 2^-8 and b 2^-16 (2^-8 + 2^-16 lies
half a step of eight bits above 2^-8, whose neighbour is the even one).  Products of two such, but for those of a second with
a third term and of two third ones, are multiples of 2^-16, and sums of 64 of them below 2^7: exact in 24 bits in
any order, also less a reference of such a sum.  So a score is off by the products that are left out alone."""
import numpy as np

HEAD = 64


def operands(rng, shape):
    a = rng.integers(0, 2, shape)
    b = rng.integers(0, 2, shape) * a
    return rng.choice([-1.0, 1.0], shape) * (1 + a * 2.0 ** -8 + b * 2.0 ** -16)


def terms(x, n=3):
    """x (24 bits) as n bf16 terms: the top eight bits, then what is left, rounded to eight."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(x)
    out = [np.ldexp(np.trunc(np.ldexp(m, 8)), e - 8)]
    for _ in range(n - 1):
        m, e = np.frexp(x - sum(out))
        out.append(np.ldexp(np.rint(np.ldexp(m, 8)), e - 8))
    return out


KEPT = [(0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0)]


def product(x, y, kept=KEPT, n=(3, 3)):
    """sum over the last axis of x y as those pairs of terms."""
    s, t = terms(x, n[0]), terms(y, n[1])
    return sum((s[i] * t[j]).sum(-1) for i, j in kept if i < n[0] and j < n[1])


def left_out(x, y):
    s, t = terms(np.abs(x)), terms(np.abs(y))
    return (s[1] * t[2] + s[2] * t[1] + s[2] * t[2]).sum(-1)


def exponent_error(d):
    """exp(s - max) of s - max = -d as a power of two: the rounding of d log2(e), at most 2^-24 of it, and of the factor log2(e) / 8,
    2^-25, then an ulp, 2^-23."""
    return np.log(2) * 1.5 * 2.0 ** -24 * d * np.log2(np.e) + 2.0 ** -23


# ---------------------------------------------------------------- scores: values +1 and -1

def score_case(rng, pairs, exact_keys=False):
    """q [pairs, 64], k [pairs, 2, 64]; exact_keys: of one term (+-1, +-1.5)."""
    q = operands(rng, (pairs, HEAD))
    k = rng.choice([-1.5, -1.0, 1.0, 1.5], (pairs, 2, HEAD)) if exact_keys else operands(rng, (pairs, 2, HEAD))
    return q, k


def score_result(q, k, scores=None):
    """(p0 - p1) / (p0 + p1) of the row that sees both keys."""
    s = (k @ q[..., None])[..., 0] if scores is None else scores
    return np.tanh((s[:, 0] - s[:, 1]) / 16)


def score_bound(q, k):
    """The difference of the scores is off by what both products leave out and by the error of the smaller probability (the other is 1),
    the result by at most half of that; the sums, the inverse and the product round six values of at most 1."""
    s = (k @ q[..., None])[..., 0] / 8
    return (left_out(q[:, None], k).sum(-1) / 8 + exponent_error(np.abs(s[:, 0] - s[:, 1]))) / 2 + 6 * 2.0 ** -24


# ---------------------------------------------------------------- values: scores d and 0

def value_case(rng, pairs):
    """d [pairs]: the second key's score less the first's, multiples of 1 / 64; v [pairs, 2, 64]."""
    return rng.integers(-128, 129, pairs) / 64, operands(rng, (pairs, 2, HEAD))


def value_result(d, v, kept=KEPT, n=(3, 3)):
    """In 64 bits, or with 24-bit probabilities and values as terms."""
    p = np.exp(np.stack([np.zeros_like(d), d], 1) - np.maximum(d, 0)[:, None])
    if kept is not KEPT or n != (3, 3):
        p = p.astype(np.float32).astype(np.float64)
        return product(p[:, None], v.swapaxes(1, 2), kept, n) / p.sum(1)[:, None]
    return (p[:, None] @ v)[:, 0] / p.sum(1)[:, None]


def value_bound(d, v):
    """The smaller probability's error moves the result by at most a quarter of it times the values' distance (below 2.02); the products
    leave out 2^-22 of the mean |v| (below 1.01); the twelve products, the sum of probabilities, its inverse and the
    last product are 15 roundings of at most 1.01."""
    return exponent_error(np.abs(d))[:, None] * 2.02 / 4 + (2.0 ** -22 + 15 * 2.0 ** -24) * 1.01
