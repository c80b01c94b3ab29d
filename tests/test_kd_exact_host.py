"""What the tests of single entries would see: mistakes planted in their own definition, on the host."""
import numpy as np

import kd_exact as ex


def test_entries_left_out_show():
    """An entry that is missing from the sums of the distillation's gradient is off by its own share, tens of bounds and more."""
    rng = np.random.default_rng(1)
    for K, d, T in ((256, 4096, 1.0), (1024, 2056, 1.3), (65, 8200, 1.0), (9, 4096, 0.5)):
        p = ex.one_each(rng, 3, K, d)
        _, dh, bound = ex.one_each_result(*p, T)
        for gone in ([K - 1], range(K - min(8, K // 4), K), [int(rng.integers(K))]):
            keep = np.ones(K, bool)
            keep[list(gone)] = False
            _, other, _ = ex.one_each_result(*p, T, keep=keep)
            at = p[2][:, list(gone)]
            far = np.abs(other - dh)[np.arange(3)[:, None], at] / bound[np.arange(3)[:, None], at]
            assert (far.max(1) > 10).all()
