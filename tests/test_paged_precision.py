"""How far roundings of the paged attention may carry a result, and that the limits tell one way of rounding from another (no GPU).

A weight p of a row is held as bf16 terms.  What they leave of it, d relative to the weight, moves the row by
  o' - o = sum_j p_j d_j (v_j - o) / (1 + sum_j p_j d_j)       where the denominator sums the terms,
  o' - o = sum_j p_j d_j v_j                                   where it sums the weights as they were,
so an element is off by max|d| times SPREAD = sum_j p_j |v_j - o|, or times sum_j p_j |v_j|, at most.  The terms leave
  one   (rounded)                          |d| <= 2^-8
  two   (upper bits, rest rounded)         |d| <= 2^-16
  three                                    |d| <= 2^-24
In a 2-norm over rows of many independent roundings the largest d is not what counts but their root mean square: a rounding to 8 bits is
spread evenly over a step, and over the mantissas of a weight that leaves 2^-7 / 12^0.5 * 0.735 = 1.66e-3 of it (0.735: the root mean square of 1 / m
for m in [1, 2) evenly in its logarithm); with two terms 5e-6 (their first one cuts, so that the rest is up to
2^-7), and with three what fp32 arithmetic leaves: scores of
ordinary size (sums of some 100 products of up to 16, 1.5e-7 of a weight), the exponent (a product and a sum of up to 16, 2e-7), sums over keys (up to
200 roundings, 3e-7): 6e-7 together at most for what the tests have."""
import numpy as np

THREE_TERMS = 1.5e-6      # 2.5 times what fp32 arithmetic leaves
TWO_TERMS = 1.2e-5        # 2.4 times what two terms leave
ONE_TERM = 2.0 ** -9      # 1.2 times what one term leaves
ONE_TERM_BF16 = 2.7e-3    # ... with an output rounded to bf16 as well: 2^0.5 * 1.66e-3, 1.15 times that


def attention(q, k, v, first, fa, n_sink, window):
    """float64 rows of queries [n, hq, d] at positions first .., and the spread of each element."""
    n, hq, d = q.shape
    grp = hq // k.shape[1]
    i, j = first + np.arange(n)[:, None], np.arange(len(k))[None]
    seen = (j <= i) & ((j < n_sink) | (i - j < window) | bool(fa))
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(hq):
        s = np.where(seen, q[:, h] @ k[:, h // grp].T / np.sqrt(d), -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        vh = v[:, h // grp]
        out[:, h] = p @ vh
        for r in range(n):
            spread[r, h] = p[r] @ np.abs(vh - out[r, h])
    return out, spread


def rel(got, ref):
    return float(np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()))


def to_bf16(x):
    b = np.asarray(x, np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32)


def in_terms(x, terms):
    """The bf16 terms of fp32 weights, added up: the upper bits of what is left, the last one rounded."""
    left, total = np.asarray(x, np.float32), np.zeros(np.shape(x))
    for t in range(terms):
        part = (left.view(np.uint32) & 0xFFFF0000).view(np.float32) if t < terms - 1 else to_bf16(left)
        total += part
        left = left - part
    return total


def rounded_rows(terms, of_terms, bf16_values=False, seed=0):
    """Rows of attention with the weights rounded so, and as they are; the denominator sums the terms or the weights."""
    rng = np.random.default_rng(seed)
    p = np.exp2(rng.standard_normal((64, 300)) * 1.5).astype(np.float32)
    v = (rng.standard_normal((300, 128)) * np.exp2(rng.uniform(0, 1, (300, 1)))).astype(np.float32)
    w = in_terms(p, terms)
    vv = to_bf16(v) if bf16_values else v
    den = (w if of_terms else p.astype(np.float64)).sum(1, keepdims=True)
    return w @ vv.astype(np.float64) / den, p.astype(np.float64) @ v / p.astype(np.float64).sum(1, keepdims=True)


def test_terms_leave_what_is_said():
    x = np.exp2(np.random.default_rng(1).uniform(-20, 20, 100000)).astype(np.float32)
    for terms, most in ((1, 2.0 ** -8), (2, 2.0 ** -16), (3, 2.0 ** -24)):
        assert (np.abs(in_terms(x, terms) - x) <= most * x).all()


def test_limits_tell_one_way_of_rounding_from_another():
    for seed in range(4):
        one, two, three = (rel(*rounded_rows(t, t == 1, seed=seed)) for t in (1, 2, 3))
        assert three < THREE_TERMS / 10 and THREE_TERMS < two / 2 and two < TWO_TERMS / 2 and TWO_TERMS < one / 10 and one < ONE_TERM / 1.1
        assert rel(*rounded_rows(1, True, True, seed=seed)) > ONE_TERM     # values rounded as well
        assert rel(*rounded_rows(1, False, seed=seed)) < ONE_TERM
