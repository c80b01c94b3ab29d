"""Low-rank adapters to the bit: whole numbers, whose sums are exact in any order, so that no row, step, run's end or part of h can go
missing unseen; and shares of y and dx that cancel but for the last of 24 bits."""
import numpy as np
import pytest

import adapt_exact as ex

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.to("cuda", dtype or t.dtype)


def i32(x):
    import torch
    return torch.tensor([int(v) for v in x], dtype=torch.int32, device="cuda")


SHAPES = [
    # rows, adapters, n, r, d_in, d_out
    ([1], [0], 1, 32, 4096, 4096),
    ([1] * 64, [i % 16 for i in range(64)], 16, 32, 1032, 520),
    ([1] * 70, [(i * 3) % 7 - 1 for i in range(70)], 6, 8, 256, 128),
    ([16, 17, 15, 32, 33, 31, 64, 65], [0, 1, 0, 2, 9, 1, 0, 2], 3, 40, 1000, 136),
    ([700, 3, 0, 450, 41], [0, 1, 2, 0, -1], 3, 24, 136, 2056),
    ([600, 500, 601, 433, 37, 700], [1, 1, 1, 1, 4, 0], 5, 64, 136, 200),
    ([600, 500, 601, 433, 37, 700], [1, 1, 1, 1, 4, 0], 5, 8, 200, 136),
    ([6] * 32, [s % 16 for s in range(32)], 16, 32, 1024, 1024),
    ([i % 90 for i in range(150)], [(i * 5) % 10 - 1 for i in range(150)], 9, 16, 128, 192),
    ([48] * 200, [i // 9 % 4 - 1 for i in range(200)], 3, 40, 64, 72),
    ([1, 2, 3, 0] * 1100, [i // 7 % 6 - 1 for i in range(4400)], 5, 16, 64, 72),
    ([9000], [0], 1, 32, 64, 72),
    ([4000, 5001, 17], [1, 0, 1], 2, 8, 4096, 4096),
    ([4000, 5001, 17], [1, 0, 1], 2, 32, 4096, 4096),
    ([4000, 5001, 17], [1, 0, 1], 2, 40, 4096, 1032),
    ([4000, 5001, 17], [1, 0, 1], 2, 64, 4096, 4096),
    ([9000], [0], 1, 64, 2056, 1032),
]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_whole_numbers(ev, shape):
    """x, dy, A and B are -1, 0 or 1 and scales powers of two: |h| <= d, and sums of |g x| stay below 2^24.  y and dx are the nearest bf16 numbers."""
    import torch
    rows, adapter, n, r, d_in, d_out = SHAPES[shape]
    rng = np.random.default_rng(shape)
    lead, tail = shape % 3, shape % 2
    off = np.concatenate([[0], np.cumsum(rows)]) + lead
    T = int(off[-1]) + tail
    bf16 = torch.bfloat16
    x, dy, A, B = (dev(ex.whole(rng, *s), bf16) for s in ((T, d_in), (T, d_out), (n, r, d_in), (n, d_out, r)))
    y0, dx0 = (dev(rng.integers(-100, 101, size=s).astype(np.float32), bf16) for s in ((T, d_out), (T, d_in)))
    scale = dev(np.float32(rng.choice([0.5, 1.0, -1.0, 2.0], size=n)))
    bank, toff, tad = ev.LoraBank(A, B, scale), i32(off), i32(adapter)
    wy, wh, wA, wB, wx = ex.lora(x, dy, A, B, scale.tolist(), off, adapter, y0, dx0)
    for magnitude in (wy, wh, wA, wB, wx):                           # (far below 2^24, and so are the sums of magnitudes: they grow as the root's square)
        assert float(magnitude.abs().max()) < 2.0 ** 20
    y, dx = y0.clone(), dx0.clone()
    h = ev.lora_forward(x, bank, toff, tad, y, keep=True)
    assert torch.equal(h.double(), wh)
    assert torch.equal(y, wy.float().to(bf16))
    for kept in (h, None):
        dx = dx0.clone()
        dA, dB = ev.lora_backward(x, dy, bank, toff, tad, h=kept, dx=dx)
        assert torch.equal(dA.double(), wA) and torch.equal(dB.double(), wB)
        assert torch.equal(dx, wx.float().to(bf16))
    outs = [torch.full_like(t, float("nan")) for t in (dA, dB)]
    ev.lora_backward(x, dy, bank, toff, tad, h=h, out_da=outs[0], out_db=outs[1])
    assert torch.equal(outs[0], dA) and torch.equal(outs[1], dB)


@pytest.mark.parametrize("r,d", [(8, 64), (16, 520), (24, 136), (32, 1024), (40, 264), (64, 512)])
@pytest.mark.parametrize("rows", [[1], [5, 40], [1] * 64, [3000, 2200], [40] * 200])
def test_the_last_bits_of_h(ev, r, d, rows):
    """Two ranks' shares of y, and of dx, cancel but for the lower 8 of h's 24 bits."""
    import torch
    rng = np.random.default_rng(r + len(rows))
    n, T = 2, sum(rows)
    off, adapter = np.concatenate([[0], np.cumsum(rows)]), [s % 2 for s in range(len(rows))]
    x, down, up, left = ex.cancelling(rng, T, n, r, d)
    which = np.repeat(adapter, rows)
    want = dev(left[which, np.arange(T)] * np.where(which, 2.0, 1.0)[:, None], torch.bfloat16)
    bf16, scale, toff, tad = torch.bfloat16, dev(np.float32([1, 2])), i32(off), i32(adapter)
    x, down, up = dev(x, bf16), dev(down, bf16), dev(up, bf16)
    y = torch.zeros(T, d, dtype=bf16, device="cuda")
    ev.lora_forward(x, ev.LoraBank(down, up.transpose(1, 2).contiguous(), scale), toff, tad, y)
    assert torch.equal(y, want)
    dx = torch.zeros_like(y)
    ev.lora_backward(x, x, ev.LoraBank(up, down.transpose(1, 2).contiguous(), scale), toff, tad, dx=dx)
    assert torch.equal(dx, want)


@pytest.mark.parametrize("n,r,d,per", [(1, 8, 64, 1), (5, 16, 136, 33), (3, 32, 1024, 700), (4, 40, 520, 65), (2, 64, 4096, 2500)])
def test_all_bits_of_h_in_the_gradients(ev, n, r, d, per):
    """One row of an adapter has a dy that is not zero, 1 everywhere: dB is its scale times h, all 24 bits of it."""
    import torch
    rng = np.random.default_rng(n)
    T, bf16 = n * per, torch.bfloat16
    row = [a * per + int(rng.integers(per)) for a in range(n)]
    h = dev(np.float32(rng.integers(2 ** 23, 2 ** 24, size=(r, T)) * 2.0 ** rng.integers(-40, 20, size=(r, T)) * rng.choice([-1, 1], size=(r, T))))
    dy = torch.zeros(T, d, dtype=bf16, device="cuda")
    dy[row] = 1
    x, A, B = dev(ex.whole(rng, T, d), bf16), dev(ex.whole(rng, n, r, d), bf16), dev(ex.whole(rng, n, d, r), bf16)
    scale = dev(np.float32(2.0 ** rng.integers(-3, 4, size=n)))
    dA, dB = ev.lora_backward(x, dy, ev.LoraBank(A, B, scale), i32([a * per for a in range(n + 1)]), i32(range(n)), h=h)
    for a in range(n):
        assert torch.equal(dB[a], (h[:, row[a]] * scale[a]).expand(d, r))
        assert torch.equal(dA[a], (scale[a] * B[a].float().sum(0))[:, None] * x[row[a]].float())
