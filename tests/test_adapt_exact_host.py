"""What the tests to the bit would see: mistakes planted in their own definition, on the host."""
import numpy as np
import pytest
import torch

import adapt_exact as ex


@pytest.mark.parametrize("r", [8, 40])
def test_rows_left_out_show(r):
    """The last 32 rows, or the last row, of any request: some element of both gradients of its adapter is another whole number."""
    rng = np.random.default_rng(r)
    rows, adapter, d_in, d_out = [64, 33, 100, 1, 90], [0, 1, 0, 1, 1], 72, 40
    off = np.concatenate([[0], np.cumsum(rows)])
    x, dy, A, B = (torch.from_numpy(ex.whole(rng, *s)) for s in ((off[-1], d_in), (off[-1], d_out), (2, r, d_in), (2, d_out, r)))
    zero = torch.zeros_like
    _, _, dA, dB, _ = ex.lora(x, dy, A, B, [1.0, 2.0], off, adapter, zero(dy), zero(x))
    for i, n in enumerate(rows):
        for left in {max(n - 32, 0), n - 1}:
            _, _, a, b, _ = ex.lora(x, dy, A, B, [1.0, 2.0], off, adapter, zero(dy), zero(x), drop=(i, left))
            assert float((a - dA)[adapter[i]].abs().max()) >= 1 and float((b - dB)[adapter[i]].abs().max()) >= 1
            other = 1 - adapter[i]
            assert torch.equal(a[other], dA[other]) and torch.equal(b[other], dB[other])


def test_bits_left_out_show():
    """h of 24 bits gives what is left between two ranks; of 16 bits, cut off, nothing of it."""
    rng = np.random.default_rng(0)
    x, down, up, left = ex.cancelling(rng, 7, 2, 16, 64)
    for a in range(2):
        h = x @ down[a].T
        assert h.max() < 2 ** 24 and np.array_equal(ex.cut(h, 24), h) and np.array_equal(h @ up[a], left[a]) and left[a].min() >= 128
        assert not (ex.cut(h, 16) @ up[a]).any()
        assert np.array_equal(np.float32(x), x) and np.array_equal(torch.from_numpy(x).to(torch.bfloat16).double().numpy(), x)
        assert np.array_equal(torch.from_numpy(left[a]).to(torch.bfloat16).double().numpy(), left[a])
