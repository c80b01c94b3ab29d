"""The distillation's gradient entry by entry: rows of W_lm with one number each, so that the share of every entry is read off an element of its own,
over the sizes of every variant, parted and not; temperatures and logits at the ends of fp32."""
import numpy as np
import pytest

import kd_exact as ex

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


def call(ev, h, value, support, target, weight, T, dtype):
    import torch
    W = torch.zeros(len(value), len(value), dtype=torch.bfloat16, device="cuda")
    W.diagonal().copy_(dev(value))
    return ev.kd_loss(dev(h, torch.bfloat16), W, dev(support), dev(target, torch.float32), dev(weight, torch.float32), T=T, dtype=dtype)


def check(got, draft, dh, bound, half=2.0 ** -24):
    assert np.array_equal(got[2].double().cpu().numpy(), draft)
    far = np.abs(got[1].double().cpu().numpy() - dh) - (bound + half * (np.abs(dh) + bound))
    assert (far <= 0).all(), (float(far.max()), np.argwhere(~(far <= 0))[:4])        # (nor is any NaN)


@pytest.mark.parametrize("E,K,d", [
    (1, 60, 64), (600, 9, 64), (5, 256, 512), (520, 33, 136), (40, 256, 1000), (3, 512, 1032), (700, 24, 648), (4, 1024, 2048), (600, 17, 1544),      # a row to a wavefront
    (1, 256, 4096), (2, 1024, 2056), (4, 9, 4096), (400, 256, 4096), (390, 37, 2056),                # a row to the workgroup; the last three not parted
    (109, 256, 4096), (150, 256, 4096), (256, 130, 4096), (192, 256, 4096), (110, 33, 2504),         # three workgroups to a unit, or two
    (1, 256, 4104), (5, 100, 4104), (2, 65, 8192), (520, 21, 5000), (2, 65, 8200), (3, 20, 16384), (260, 33, 8200), (1, 7, 12296)])
@pytest.mark.parametrize("fp32", [True, False])
def test_entry_by_entry(ev, E, K, d, fp32):
    import torch
    p = ex.one_each(np.random.default_rng(E + K + d), E, K, d)
    for T in (1.0, 0.5):
        got = call(ev, *p, T, torch.float32 if fp32 else torch.bfloat16)
        check(got, *ex.one_each_result(*p, T), 2.0 ** -24 if fp32 else 2.0 ** -8)


@pytest.mark.parametrize("E,K,d", [(6, 60, 64), (600, 60, 1000), (4, 100, 4096), (400, 9, 4096), (3, 40, 8200)])
@pytest.mark.parametrize("T", [2.0 ** -126, 1e-37, 1e-30, 0.01, 50.0, 1e30])
def test_temperatures(ev, E, K, d, T):
    """Down to where 1 / T is only just finite: the largest logit alone, or the largest ones, alike."""
    import torch
    T = float(np.float32(T))
    p = ex.one_each(np.random.default_rng(K), E, K, d)
    got = call(ev, *p, T, torch.float32)
    check(got, *ex.one_each_result(*p, T))
    assert T > 50 or (not got[0].isnan().any() and (got[0] >= 0).all())


@pytest.mark.parametrize("E,K,d", [(3, 60, 64), (600, 40, 64), (600, 20, 648), (2, 256, 1000), (600, 24, 2000), (3, 100, 4096), (400, 9, 4096), (3, 40, 8200)])
def test_logits_of_minus_infinity(ev, E, K, d):
    """Sums past fp32's range: shares of zero, wherever they come, the first entries of every part and turn among them."""
    import torch
    rng = np.random.default_rng(d)
    h, value, support, target, weight = ex.one_each(rng, E, K, d)
    value[rng.random(d) < 0.7] = -4.0
    gone = (rng.random((E, d)) < 0.7) & (value == -4)                # elements whose logits are -2^129
    gone[0, support[0, :8]], value[support[0, :8]] = True, -4.0
    gone[np.arange(E), support[:, K - 1]] = False
    h[gone] = 2.0 ** 127
    inside = ~gone[np.arange(E)[:, None], support]
    assert not inside[0, :8].any() and inside.any(1).all()
    target = np.where(inside, target, -np.inf).astype(np.float32)    # (nor does the target want them)
    got = call(ev, h, value, support, target, weight, 1.0, torch.float32)
    draft, dh, bound = ex.one_each_result(h, value, support, target, weight, 1.0)
    check(got, np.where(inside, draft, -np.inf), dh, bound)
    assert got[0].isfinite().all()
    target[0, 0] = 1.0                                               # one that it wants: an infinite loss, and no NaN
    got = call(ev, h, value, support, target, weight, 1.0, torch.float32)
    assert got[0][0] == float("inf") and got[0][1:].isfinite().all() and got[1].isfinite().all()
