"""What the tolerances of attention_bounds.py let through: nothing that is wrong in as much as one block of 32 tokens."""
import numpy as np
import pytest

import attention_bounds as bounds
import decode_reference as ref


@pytest.mark.parametrize("kind,type,dim", [("e4m3", "bf16", 128), ("int8", "fp16", 64)])
@pytest.mark.parametrize("rows", [1, 9])
def test_a_wrong_block_is_seen(kind, type, dim, rows):
    """K or V of any block of a long sequence taken from the block behind it."""
    import torch
    rng = np.random.default_rng(rows + dim)
    lens, page = [5000], 64
    c = ref.Cache(80, page, 1, dim, kind, rng)
    table = rng.permutation(80)[:79].reshape(1, 79)
    bounds.code_by_place(c, table)
    q = rng.standard_normal((rows, 2, dim))
    off = [0, rows]
    good = bounds.attention(c, q, table, lens, off, 2, type)
    dtype = torch.bfloat16 if type == "bf16" else torch.float16

    def rounded(x):
        return torch.from_numpy(x).to(dtype).double().numpy()

    assert bounds.differs(rounded(good[0]), good[1], good) is None
    blocks = (lens[0] - rows) // ref.BLOCK                       # (those that all rows see as a whole)
    for b in range(0, blocks - 1, 7 if rows > 1 else 3):
        for part in (0, 1):
            def change(s, k, v, b=b, part=part):
                x = (k, v)[part]
                x[32 * b:32 * b + 32] = x[32 * b + 32:32 * b + 64].copy()
            bad = bounds.attention(c, q, table, lens, off, 2, type, change=change)
            assert bounds.differs(rounded(bad[0]), bad[1], good) is not None, (b, part)


def test_a_missing_token_is_seen():
    """A token too few or too many at the end of what a row sees."""
    rng = np.random.default_rng(3)
    c = ref.Cache(40, 64, 1, 64, "e4m3", rng)
    table = rng.permutation(40).reshape(1, 40)
    bounds.code_by_place(c, table)
    q = rng.standard_normal((1, 4, 64))
    for n in (33, 500, 2500):
        good = bounds.attention(c, q, table, [n], [0, 1], 4, "bf16")
        for other in (n - 1, n + 1):
            bad = bounds.attention(c, q, table, [other], [0, 1], 4, "bf16")
            assert bounds.differs(bad[0], bad[1], good) is not None, (n, other)
