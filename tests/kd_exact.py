"""Distillation problems with one number in every row of W_lm, so that every entry of a support is read off an element of its own."""
import numpy as np


def one_each(rng, E, K, d):
    """Row i of W_lm has one number, value[i] (1 or 2), at element i, and no two entries of an event are alike: (h, value, support, target, weight).
    A logit is one product, exact."""
    assert K <= d
    value = rng.integers(1, 3, size=d).astype(np.float64)
    h = rng.integers(-64, 65, size=(E, d)) / 16.0                    # (bf16 numbers)
    support = np.stack([rng.permutation(d)[:K] for _ in range(E)]).astype(np.int32)
    target = np.float32(rng.normal(size=(E, K)) * 2)
    return h, value, support, target, np.float32(0.25 + rng.random(E))


def one_each_result(h, value, support, target, weight, T, keep=None):
    """(draft, gradient, bound of it) in 64 bits; keep: the entries (by number) that are in the sums, all of them if None."""
    U = 2.0 ** -24
    E, K = support.shape
    draft = h[np.arange(E)[:, None], support] * value[support]
    t = target.astype(np.float64)
    b, a = (t.max(1, keepdims=True) - t) / T, (draft.max(1, keepdims=True) - draft) / T
    p, q = np.exp(-b), np.exp(-a)
    if keep is not None:
        q = np.where(keep, q, 0.0)
    p, q = p / p.sum(1, keepdims=True), q / q.sum(1, keepdims=True)
    if keep is not None:
        p = np.where(keep, p, 0.0)
    at = (np.arange(E)[:, None], support)
    dh, bound = np.zeros(h.shape), np.zeros(h.shape)
    scale = weight.astype(np.float64)[:, None] * T * value[support]
    dh[at] = scale * (q - p)
    # An argument is a difference, divided: three roundings of itself, a function of it right to four; a share is divided by a sum of K, whose terms'
    # arguments are off likewise (x exp(-x) < 1 of them); both may have been scaled down anew at every entry; a few products.
    few = (6 * K + 32) * U
    bound[at] = np.abs(scale) * (q * (few + 4 * U * np.minimum(a, 1e3)) + p * (few + 4 * U * np.minimum(b, 1e3))) + 2.0 ** -146
    return draft, dh, bound
