"""Which places in memory meet, against their bytes one by one."""
import random

import pytest


def bytes_of(p):
    lo, hi, row, step, _ = p
    return {b for at in range(lo, hi, step) for b in range(at, min(at + row, hi))} if hi > lo else set()


def place(rng, strides):
    rows, step = rng.randrange(0, 5), rng.choice(strides)
    row = rng.randrange(1, step + 1)
    lo = rng.randrange(100, 160)
    if rng.random() < 0.3 or rows < 2:                               # contiguous
        n = rng.randrange(0, 60)
        return lo, lo + n, n, n, "x"
    return lo, lo + (rows - 1) * step + row, row, step, "x"


def test_meet():
    from paper_2605_27390_amd.adapt import _meet
    rng = random.Random(0)
    seen = [0, 0]
    for _ in range(20000):
        a, b = place(rng, [24]), place(rng, [24])                    # one stride, or one row
        want = bool(bytes_of(a) & bytes_of(b))
        assert _meet(a, b) == _meet(b, a) == want, (a, b)
        seen[want] += 1
    assert min(seen) > 2000
    for _ in range(5000):                                            # others may be refused, and never missed
        a, b = place(rng, [16, 24, 40]), place(rng, [16, 24, 40])
        assert _meet(a, b) or not bytes_of(a) & bytes_of(b), (a, b)


def test_many_places():
    from paper_2605_27390_amd.adapt import _refuse_all
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(5000):
        def some(n):
            return [(lo, lo + k, k, k, "x") for lo, k in ((rng.randrange(0, 200), rng.randrange(0, 25)) for _ in range(n))]
        written, read = some(rng.randrange(1, 4)), some(rng.randrange(0, 4))
        want = any(bytes_of(a) & bytes_of(b) for i, a in enumerate(written) for b in written[:i] + read)
        seen[want] += 1
        if want:
            with pytest.raises(ValueError, match="overlaps"):
                _refuse_all(written, read)
        else:
            _refuse_all(written, read)
    assert min(seen) > 500
