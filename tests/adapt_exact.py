"""Problems of the adapters whose results the kernels have to meet to the bit: whole numbers, so that every product and every sum in fp32 is exact in any
order, with the definition in 64-bit torch on any device."""
import numpy as np
import torch


def requests(row_off, adapter, T, n):
    """(rows, adapter) of the requests that have one."""
    for s, a in enumerate(adapter):
        r0 = min(max(int(row_off[s]), 0), T)
        r1 = min(max(int(row_off[s + 1]), r0), T)
        if 0 <= a < n and r1 > r0:
            yield slice(r0, r1), int(a)


def whole(rng, *shape):
    """-1, 0 and 1."""
    return rng.integers(-1, 2, size=shape).astype(np.float32)


def lora(x, dy, A, B, scale, row_off, adapter, y, dx, drop=None):
    """(y, h, dA, dB, dx) in 64 bits; drop = (request, row): rows of that request from there on are left out of the gradients."""
    T, (n, r, d_in) = x.shape[0], A.shape
    y, dx = y.double(), dx.double()
    h = torch.zeros((r, T), dtype=torch.float64, device=x.device)
    dA, dB = torch.zeros(A.shape, dtype=torch.float64, device=x.device), torch.zeros(B.shape, dtype=torch.float64, device=x.device)
    for i, (rows, a) in enumerate(requests(row_off, adapter, T, n)):
        xr, gr, Aa, Ba, s = x[rows].double(), dy[rows].double(), A[a].double(), B[a].double(), float(scale[a])
        hr = xr @ Aa.t()
        g = s * (gr @ Ba)
        h[:, rows] = hr.t()
        y[rows] += s * (hr @ Ba.t())
        dx[rows] += g @ Aa
        if drop is not None and drop[0] == i:
            xr, gr, hr, g = xr[:drop[1]], gr[:drop[1]], hr[:drop[1]], g[:drop[1]]
        dA[a] += g.t() @ xr
        dB[a] += s * (gr.t() @ hr)
    return y, h, dA, dB, dx


def cancelling(rng, T, n, r, d):
    """(x [T, d], down [n, r, d], up [n, r, d], left [n, T, d]): h = x down^T has 24 bits in every even rank, the odd one after it the upper 16 of
    them, and h up is what is left between the two, the lower 8 bits, in every column that pair's.  Every pair has three elements of x of its own."""
    pairs = r // 2
    assert d >= 3 * pairs
    x = np.zeros((T, d))
    parts = rng.integers(128, 256, size=(T, pairs, 3)) * np.array([65536, 256, 1])
    x[:, :3 * pairs] = parts.reshape(T, 3 * pairs)
    down, up, left = np.zeros((n, r, d)), np.zeros((n, r, d)), np.zeros((n, T, d))
    for a in range(n):
        for k in range(pairs):
            down[a, 2 * k, 3 * k:3 * k + 3], down[a, 2 * k + 1, 3 * k:3 * k + 2] = 1, 1
        of = (np.arange(d) * (2 * a + 1) + a) % pairs
        up[a, 2 * of, np.arange(d)], up[a, 2 * of + 1, np.arange(d)] = 1, -1
        left[a] = parts[:, of, 2]
    return x, down, up, left


def cut(h, bits):
    """h with so many bits, the others cut off."""
    f, e = np.frexp(h)
    return np.ldexp(np.trunc(f * 2.0 ** bits), e - bits)
