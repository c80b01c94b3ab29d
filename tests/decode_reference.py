"""Plain implementations, in 64 bits on the host, of the 8-bit cache, the attention over it and the sampler."""
import numpy as np

BLOCK = 32


def e4m3_values():
    """The 256 codes of 4 exponent and 3 mantissa bits (bias 7, no infinities, 0x7f is NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


E4M3 = e4m3_values()


def decode(codes, kind):
    codes = np.asarray(codes, dtype=np.uint8)
    if kind == "e4m3":
        return E4M3[codes]
    v = codes.view(np.int8).astype(np.float64)
    return np.where(codes == 128, np.nan, v)


def encode(y, kind):
    """Codes of values that are divided by the scale already."""
    y = np.asarray(y, dtype=np.float64)
    nan = np.isnan(y)
    y = np.where(nan, 0.0, y)
    if kind == "int8":
        c = np.rint(np.clip(y, -127, 127)).astype(np.int64) & 255
        return np.where(nan, 128, c).astype(np.uint8)
    a = np.minimum(np.abs(y), 448.0)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    q = np.rint(a / 2.0 ** (e - 3)) * 2.0 ** (e - 3)                     # nearest, ties to even
    pos = E4M3[:127]
    c = np.searchsorted(pos, q)
    assert np.array_equal(pos[c], q)
    c = c + np.where(np.signbit(y), 128, 0)
    return np.where(nan, 127, c).astype(np.uint8)


def scale_of(amax, kind):
    if kind == "int8":
        return max(np.float32(amax) / np.float32(127), np.float32(2.0 ** -100))
    e = -100
    while e < 120 and amax > 448.0 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def block_bytes(k, v):
    """Codes of a block, [32 tokens, dim] each, in the order of the cache: 2 x 32 dim bytes."""
    D = k.shape[1]
    ok, ov = np.empty(32 * D, np.uint8), np.empty(32 * D, np.uint8)
    for t in range(32):
        for d in range(D):
            s, r = divmod(d, 32)
            ok[s * 1024 + (r // 16) * 512 + t * 16 + r % 16] = k[t, d]
            a, g, i = t // 8, (t // 4) % 2, t % 4
            ov[s * 1024 + g * 512 + r * 16 + 4 * a + i] = v[t, d]
    return np.stack([ok, ov])


def block_codes(b):
    """The other way: [2, 32 dim] bytes to K and V codes [32, dim]."""
    D = b.shape[1] // 32
    at = np.arange(32 * D, dtype=np.int64).reshape(32, D)
    k_at, v_at = np.empty((32, D), np.int64), np.empty((32, D), np.int64)
    t, d = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
    s, r = d // 32, d % 32
    k_at[...] = s * 1024 + (r // 16) * 512 + t * 16 + r % 16
    v_at[...] = s * 1024 + ((t // 4) % 2) * 512 + r * 16 + 4 * (t // 8) + t % 4
    del at
    return b[0][k_at], b[1][v_at]


class Cache:
    """A cache on the host: bytes and scales as in include/evospec_decode.h."""

    def __init__(self, pages, page, heads, dim, kind, rng=None):
        self.pages, self.page, self.heads, self.dim, self.kind = pages, page, heads, dim, kind
        shape = (pages, heads, page // BLOCK, 2)
        if rng is None:
            self.data = np.full(shape + (BLOCK * dim,), 0x7F if kind == "e4m3" else 0x80, np.uint8)   # all NaN
            self.scales = np.full(shape, np.nan, np.float32)
        else:
            x = rng.standard_normal(shape + (BLOCK * dim,))
            if kind == "e4m3":
                self.data = encode(x * 64, kind)
                self.scales = (2.0 ** rng.integers(-8, -4, shape)).astype(np.float32)
            else:
                self.data = encode(x * 28, kind)
                self.scales = ((0.5 + rng.random(shape)) / 28).astype(np.float32)

    def place(self, table, s, block):
        """(page, block of it) or None."""
        per = self.page // BLOCK
        if block // per >= table.shape[1]:
            return None
        p = int(table[s, block // per])
        return (p, block % per) if 0 <= p < self.pages else None

    def write(self, k, v, table, starts, row_off):
        """k, v: float32 arrays [T, heads, dim] (exact values of the callers' type)."""
        for s in range(len(starts)):
            n, a = row_off[s + 1] - row_off[s], int(starts[s])
            for block in range(a // BLOCK, (a + n + BLOCK - 1) // BLOCK if n else 0):
                at = self.place(table, s, block)
                if at is None:
                    continue
                t0 = block * BLOCK
                first, last = max(0, a - t0), min(BLOCK, a + n - t0)
                for h in range(self.heads):
                    old = block_codes(self.data[at[0], h, at[1]])
                    new = []
                    for w, x in enumerate((k, v)):
                        rows = x[row_off[s] + t0 + first - a:row_off[s] + t0 + last - a, h].astype(np.float32)
                        finite = np.isfinite(rows)
                        sc = scale_of(np.abs(rows[finite]).max(initial=0.0), self.kind)
                        nan = np.isnan(rows).any()
                        codes = old[w].copy()
                        if first:
                            so = self.scales[at[0], h, at[1], w]
                            nan |= np.signbit(so)
                            so = abs(so)
                            sc = max(sc, so)
                            if sc != so:
                                y = decode(codes[:first], self.kind).astype(np.float32) * so
                                codes[:first] = encode(y / sc, self.kind)
                        with np.errstate(over="ignore"):
                            codes[first:last] = encode((rows / sc).astype(np.float32), self.kind)
                        self.scales[at[0], h, at[1], w] = -sc if nan else sc
                        new.append(codes)
                    self.data[at[0], h, at[1]] = block_bytes(*new)

    def values(self, table, s, n):
        """K, V [n, heads, dim] of the first n tokens in 64 bits, and which of them have a page."""
        k, v = np.zeros((2, n, self.heads, self.dim))
        there = np.zeros(n, bool)
        for block in range((n + BLOCK - 1) // BLOCK):
            at = self.place(table, s, block)
            if at is None:
                continue
            t0, t1 = block * BLOCK, min(n, block * BLOCK + BLOCK)
            there[t0:t1] = True
            for h in range(self.heads):
                ck, cv = block_codes(self.data[at[0], h, at[1]])
                sc = np.abs(self.scales[at[0], h, at[1]].astype(np.float64))
                k[t0:t1, h] = (decode(ck, self.kind) * sc[0])[:t1 - t0]
                v[t0:t1, h] = (decode(cv, self.kind) * sc[1])[:t1 - t0]
        return k, v, there


def attention(cache, q, table, lens, row_off, group, tree, scale):
    """(out, lse, weight, score): out and lse in 64 bits; weight = sum softmax |v| per element and score = the largest
    sum of |q k| scale of a row, in which errors are measured."""
    T, heads, D = q.shape
    out, lse = np.zeros((T, heads, D)), np.full((T, heads), -np.inf)
    weight, score = np.zeros((T, heads, D)), np.zeros((T, heads))
    for s in range(len(lens)):
        n = row_off[s + 1] - row_off[s]
        L = max(0, min(int(lens[s]), table.shape[1] * cache.page))
        base = int(L - n)
        k, v, there = cache.values(table, s, L)
        t = np.arange(L)
        for i in range(n):
            r = row_off[s] + i
            if tree is None:
                seen = t <= base + i
            else:
                seen = (t < base) | np.array([t_ >= base and (int(tree[r]) >> (t_ - base)) & 1 == 1 for t_ in range(L)], dtype=bool)
            seen &= there
            if not seen.any():
                continue
            for a in range(heads):
                h = a // group
                x = k[seen, h] @ q[r, a] * scale
                score[r, a] = (np.abs(k[seen, h]) @ np.abs(q[r, a])).max() * scale
                m = x.max()
                p = np.exp(x - m)
                lse[r, a] = m + np.log(p.sum())
                p /= p.sum()
                out[r, a] = p @ v[seen, h]
                weight[r, a] = p @ np.abs(v[seen, h])
    return out, lse, weight, score


def sample(z, u, temperature=None, top_k=None, top_p=None, min_p=None, ids=None):
    """(ids, logprob, margin): margin is how far u's place is from the nearest border, in shares of the kept tokens."""
    M, V = z.shape
    out, lp, margin = np.full(M, -1), np.full(M, np.nan), np.full(M, np.inf)
    for m in range(M):
        row = z[m].astype(np.float64)
        row = np.where(np.isnan(row), -np.inf, row) + 0.0
        token = np.arange(V) if ids is None else np.asarray(ids).astype(np.int64)
        at = np.flatnonzero(row > -np.inf)
        if not at.size:
            continue
        at = at[np.lexsort((token[at], -row[at]))]
        T = 1.0 if temperature is None else float(temperature[m])
        if not T > 0:
            out[m], lp[m] = token[at[0]], 0.0
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(row[at] == row[at[0]], 1.0, np.exp((row[at] - row[at[0]]) / T))
        if top_k is not None and top_k[m] > 0:
            w = w[:top_k[m]]
        if top_p is not None and top_p[m] < 1:
            c = np.cumsum(w)
            w = w[:max(1, int((c - w < float(top_p[m]) * c[-1]).sum()))]
        if min_p is not None and min_p[m] > 0:
            w = w[:max(1, int((w >= float(min_p[m])).sum()))]
        c = np.cumsum(w)
        # tokens that weigh nothing next to the first are not drawn
        last = int((w >= 2.0 ** -44).sum()) - 1
        j = min(int((c <= float(u[m]) * c[-1]).sum()), last)
        out[m], lp[m] = token[at[j]], np.log(w[j] / c[-1])
        margin[m] = np.abs(c / c[-1] - float(u[m])).min()
    return out, lp, margin
