"""The formula of include/evospec_decode.h's attention in 64 bits, and for each output how far off it may be.

For one row, with x_j = scale q.k_j, s_j the scale of V's block of token j, c_j the codes of V, v_j = c_j s_j, w = softmax(x), A = sum w |v|:
  * a score is a sum of dim exact products in 32 bits, off by E = (dim + 8) 2^-24 max_j scale |q|.|k_j| at most; the argument of the exponential,
    t_j = x_j log2(e) + log2(s_j) minus the row's reference, is of a few such operations on numbers no larger than X = max |x| log2(e) + max |log2 s| + 1,
    and V's scale comes back by a reciprocal: B = 2^-23 (8 X + 8).  Both move a weight, and the sum of the weights, by a factor of 1 +- (E + B);
  * a weight is rounded to fp16: 2^-11 of it, or, below 2^-14 of the row's reference, 2^-25 of that.  The reference is not above max_j t_j, so in
    the output, which is divided by sum e^x, that is no more than R = 2^-25 sum_j |c_j| max_j (e^x_j s_j) / sum_j e^x_j;
  * the sums are in 32 bits.  A workgroup's four wavefronts have every fourth block each: n / 4 tokens follow one another in the output's sum, n / 8
    in that of the weights (a lane has half of a block's), and then come the wavefronts' and the workgroups' shares, 128 at most:
    N = (3 n / 8 + 320) 2^-24 for both;
  * the output is rounded to its type: eps / 2 of it.
    |out - exact| <= (|exact| + err) eps / 2 + err,  err = A (2^-11 + 2 (E + B) + N) + R
    |lse - exact| <= E + B + N + 2^-22 |lse|

A row over thousands of tokens says little about one block of them, if every block has a share in every element.  `code_by_place` leaves V
of block b of a sequence nothing but the elements d = b mod dim: each element is then the share of a few blocks, and tells them apart.
"""
import numpy as np

import decode_reference as ref

EPS = {"bf16": 2.0 ** -7, "fp16": 2.0 ** -10}


def code_by_place(cache, table):
    """Clears V of every block of every sequence but for one element in `dim` (see above)."""
    per = cache.page // ref.BLOCK
    for row in table:
        for i, page in enumerate(row):
            for j in range(per):
                for h in range(cache.heads):
                    k, v = ref.block_codes(cache.data[page, h, j])
                    d = (i * per + j) % cache.dim
                    keep = v[:, d].copy()
                    keep[keep & 0x7F == 0] = 0x21            # (no zeros among them)
                    v = np.zeros_like(v)
                    v[:, d] = keep
                    cache.data[page, h, j] = ref.block_bytes(k, v)


def sequence(cache, table, s, n):
    """K, V [n, heads, dim], V's codes and scales [n, heads(, dim)] and which tokens have a page."""
    k, v = np.zeros((2, n, cache.heads, cache.dim))
    c, sc, there = np.zeros((n, cache.heads, cache.dim)), np.ones((n, cache.heads)), np.zeros(n, bool)
    for block in range((n + ref.BLOCK - 1) // ref.BLOCK):
        at = cache.place(table, s, block)
        if at is None:
            continue
        t0, t1 = block * ref.BLOCK, min(n, (block + 1) * ref.BLOCK)
        there[t0:t1] = True
        for h in range(cache.heads):
            ck, cv = ref.block_codes(cache.data[at[0], h, at[1]])
            a = np.abs(cache.scales[at[0], h, at[1]].astype(np.float64))
            k[t0:t1, h] = (ref.decode(ck, cache.kind) * a[0])[:t1 - t0]
            c[t0:t1, h] = ref.decode(cv, cache.kind)[:t1 - t0]
            sc[t0:t1, h] = a[1]
    v = c * sc[..., None]
    return k, v, c, sc, there


def attention(cache, q, table, lens, row_off, group, type, tree=None, scale=None, change=None):
    """(out, lse, tol, lse_tol).  `change(k, v)` may spoil a sequence's K and V in place: what a kernel that is wrong would give."""
    T, heads, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    out, lse = np.zeros((T, heads, D)), np.full((T, heads), -np.inf)
    tol, lse_tol = np.zeros((T, heads, D)), np.zeros((T, heads))
    for s in range(len(lens)):
        n = row_off[s + 1] - row_off[s]
        L = max(0, min(int(lens[s]), table.shape[1] * cache.page))
        base = int(L - n)
        k, v, c, sc, there = sequence(cache, table, s, L)
        if change is not None:
            change(s, k, v)
        t = np.arange(L)
        for i in range(n):
            r = row_off[s] + i
            if tree is None:
                seen = t <= base + i
            else:
                word = int(tree[r]) & (2 ** 64 - 1)
                seen = (t < base) | np.array([b >= base and (word >> (b - base)) & 1 == 1 for b in range(L)], dtype=bool)
            seen &= there
            m = int(seen.sum())
            if not m:
                continue
            for a in range(heads):
                h = a // group
                x = k[seen, h] @ q[r, a] * scale
                top = x.max()
                p = np.exp(x - top)
                total = p.sum()
                w = p / total
                s_v = np.maximum(sc[seen, h], 2.0 ** -100)
                E = (D + 8) * 2.0 ** -24 * (np.abs(k[seen, h]) @ np.abs(q[r, a])).max() * scale
                X = np.abs(x).max() * np.log2(np.e) + np.abs(np.log2(s_v)).max() + 1
                B = 2.0 ** -23 * (8 * X + 8)
                R = 2.0 ** -25 * np.abs(c[seen, h]).sum(0) * (p * s_v).max() / total
                out[r, a], lse[r, a] = w @ v[seen, h], top + np.log(total)
                N = (3 * m / 8 + 320) * 2.0 ** -24
                err = (w @ np.abs(v[seen, h])) * (2.0 ** -11 + 2 * (E + B) + N) + R
                tol[r, a] = (np.abs(out[r, a]) + err) * EPS[type] / 2 + err
                lse_tol[r, a] = E + B + N + 2.0 ** -22 * abs(lse[r, a])
    return out, lse, tol, lse_tol


def differs(got, got_lse, want):
    """None, or where a result lies outside of what it may be."""
    out, lse, tol, lse_tol = want
    if not np.isfinite(got).all():
        return "not finite", np.argwhere(~np.isfinite(got))[0].tolist()
    off = np.abs(got - out) - tol
    if (off > 0).any():
        return "out", np.unravel_index(off.argmax(), off.shape), (np.abs(got - out) / np.maximum(tol, 1e-300)).max()
    empty = np.isneginf(lse)
    if not np.array_equal(np.isneginf(got_lse), empty):
        return "empty rows", np.argwhere(np.isneginf(got_lse) != empty)[0].tolist()
    off = np.abs(got_lse[~empty] - lse[~empty]) - lse_tol[~empty]
    return ("lse", float(off.max())) if (off > 0).any() else None
