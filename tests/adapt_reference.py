"""Plain implementations, in 64 bits on the host, of the adapters, the distillation loss and AdamW, each with a bound of what the kernels'
arithmetic may be off by.  U is half a step of fp32; a sum of n products in fp32, in any order, is off by at most n U times
the sum of their magnitudes."""
import numpy as np

U = 2.0 ** -24
BF16 = 2.0 ** -8                                                     # half a step, relative
HALF = {"bf16": BF16, "fp16": 2.0 ** -11, "fp32": U}


def bf16(x):
    """Nearest bf16 numbers, as fp64."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


# ---------------------------------------------------------------- adapters

def requests(row_off, adapter, T, n):
    """(rows, adapter) of the requests that have one."""
    for s, a in enumerate(adapter):
        r0 = min(max(row_off[s], 0), T)
        r1 = min(max(row_off[s + 1], r0), T)
        if 0 <= a < n and r1 > r0:
            yield slice(r0, r1), a


def lora_forward(x, A, B, scale, row_off, adapter, y):
    """(y, its bound, h [r, T] with NaN where no adapter is, its bound)"""
    T, (n, r, d_in) = x.shape[0], A.shape
    y, bound = y.copy(), np.zeros_like(y)
    h, hb = np.full((r, T), np.nan), np.full((r, T), np.nan)
    for rows, a in requests(row_off, adapter, T, n):
        p, mag = x[rows] @ A[a].T, np.abs(x[rows]) @ np.abs(A[a]).T
        h[:, rows], hb[:, rows] = p.T, d_in * U * mag.T
        s = 1.0 if scale is None else scale[a]
        y[rows] += s * (p @ B[a].T)
        # h in two bf16 numbers, the second one cut off: 2^-16 of it at most
        up = (2.0 ** -16 + (d_in + 2 * r + 4) * U) * abs(s) * (mag @ np.abs(B[a]).T)
        bound[rows] = BF16 * (np.abs(y[rows]) + up) + up
    return y, bound, h, hb


def lora_backward(x, dy, A, B, scale, row_off, adapter, dx):
    """(dA, bound, dB, bound, dx, bound); dx may be None"""
    T, (n, r, d_in) = x.shape[0], A.shape
    d_out = B.shape[1]
    dA, dAb, dB, dBb = np.zeros(A.shape), np.zeros(A.shape), np.zeros(B.shape), np.zeros(B.shape)
    dx = None if dx is None else dx.copy()
    dxb = None if dx is None else np.zeros_like(dx)
    for rows, a in requests(row_off, adapter, T, n):
        s = 1.0 if scale is None else scale[a]
        g, gm = s * (dy[rows] @ B[a]), abs(s) * (np.abs(dy[rows]) @ np.abs(B[a]))
        h, hm = s * (x[rows] @ A[a].T), abs(s) * (np.abs(x[rows]) @ np.abs(A[a]).T)
        dA[a] += g.T @ x[rows]
        dB[a] += dy[rows].T @ h
        # three cut parts are all of fp32's bits; three products are added for each row
        dAb[a] += (d_out + 3 * T + 40) * U * (gm.T @ np.abs(x[rows]))
        dBb[a] += (d_in + 3 * T + 40) * U * (np.abs(dy[rows]).T @ hm)
        if dx is not None:
            dx[rows] += g @ A[a]
            up = (2.0 ** -16 + (d_out + 2 * r + 4) * U) * (gm @ np.abs(A[a]))
            dxb[rows] = BF16 * (np.abs(dx[rows]) + up) + up
    return dA, dAb, dB, dBb, dx, dxb


# ---------------------------------------------------------------- distillation

def kd_loss(h, W, support, target, weight, T, half):
    """(loss, bound, dh, bound, draft, bound)"""
    E, d = h.shape
    K, V = support.shape[1], W.shape[0]
    loss, lb, dh, db = np.zeros(E), np.zeros(E), np.zeros((E, d)), np.zeros((E, d))
    draft, zb = np.full((E, K), np.nan), np.full((E, K), np.nan)
    for e in range(E):
        at = np.nonzero((support[e] >= 0) & (support[e] < V))[0]
        rows = W[support[e, at]]
        z, ez = rows @ h[e], d * U * (np.abs(rows) @ np.abs(h[e]))
        draft[e, at], zb[e, at] = z, ez
        t = target[e, at]
        if at.size == 0 or (not np.isnan(t).any() and np.max(t) == -np.inf):
            continue
        w = 1.0 if weight is None else weight[e]
        mt, mz = np.max(t), np.max(z)
        with np.errstate(invalid="ignore", divide="ignore"):
            lp = (t - mt) / T - np.log(np.sum(np.exp((t - mt) / T)))
            lq = (z - mz) / T - np.log(np.sum(np.exp((z - mz) / T)))
            p, q = np.exp(lp), np.exp(lq)
            loss[e] = w * T * T * np.sum(np.where(p > 0, p * (lp - lq), 0.0))
            dh[e] = w * T * ((q - p) @ rows)
            # the logits' errors go through q - p, twice for what is not linear; the rest is in 64 bits
            lb[e] = 2 * abs(w) * T * np.sum(np.abs(q - p) * ez) + 2 * U * abs(loss[e]) + 1e-12 * abs(w) * T * T * (1 + np.max(np.abs(lq)))
            # weights: the logits' error, a few roundings of an argument and a function of it, and a sum of K
            far = 8 * U * (np.max(np.abs(z)) + np.max(np.abs(t[np.isfinite(t)]), initial=0.0)) / T
            eq = 3 * np.max(ez) / T + (2 * K + 24) * U + far
            db[e] = abs(w) * T * (eq * ((q + p) @ np.abs(rows)))
            db[e] += half * (np.abs(dh[e]) + db[e])
    return loss, lb, dh, db, draft, zb


# ---------------------------------------------------------------- AdamW

def random_bits(place, seed, t):
    M = np.uint64(0xffffffff)
    x = (np.asarray(place, np.uint64) * np.uint64(0x9e3779b1) + np.uint64((seed * 0x85ebca6b + t * 0xc2b2ae35) & 0xffffffff)) & M
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x21f0aaad)) & M
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x735a2d97)) & M
    return (x ^ (x >> np.uint64(15))).astype(np.int64)


def scale_for(amax, largest):
    e = -100
    while e < 100 and amax > largest * 2.0 ** e:
        e += 1
    return 2.0 ** e


def grid(y, bits, bias, largest):
    """Codes of magnitudes y: on the grid of 3 mantissa bits the number below, or above where y's part of a step and the random one reach 1."""
    y = np.minimum(y, largest)
    e = np.maximum(np.floor(np.log2(np.maximum(y, 2.0 ** (1 - bias)))), 1 - bias)
    n = np.floor(y / 2.0 ** (e - 3) + bits / 65536.0)               # steps of 2^(e - 3): 8 .. 16, below 8 the numbers without exponent
    return ((e + bias - 1) * 8 + n).astype(np.int64)


def m_values(codes):
    c = np.asarray(codes, np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where((c & 127) == 127, np.nan, np.where(c >= 128, -v, v))


def v_values(codes):
    c = np.asarray(codes, np.int64)
    e, f = c >> 3, c & 7
    return np.where(e == 0, f * 2.0 ** -17, (8 + f) * 2.0 ** (e - 18.0))


def adamw(p, g, m, v, lr, t, betas, eps, weight_decay, grad_scale=1.0):
    """(p, bound, m, bound, v, bound), p before it is rounded to its type"""
    b1, b2 = betas
    g = g * grad_scale
    em = 5 * U * (b1 * np.abs(m) + (1 - b1) * np.abs(g)) + 2.0 ** -148
    ev = 6 * U * (b2 * v + (1 - b2) * g * g) + 2.0 ** -126
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    rate, den = lr / (1 - b1 ** t), np.sqrt(v / (1 - b2 ** t)) + eps
    u = rate * m / den
    new = p * (1 - lr * weight_decay) - u
    # the root and its sum with eps: relative errors of v by half, and of a function that is right to a step
    root = np.sqrt((v + ev) / (1 - b2 ** t)) - np.sqrt(np.maximum(v - ev, 0.0) / (1 - b2 ** t))
    bound = rate * em / den + np.abs(u) * (root / den + 16 * U) + 3 * U * (np.abs(p) + np.abs(u))
    return new, bound, m, em, v, ev
