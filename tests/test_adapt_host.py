"""Host-only checks of include/evospec_adapt.h: sizes, and refusals before anything touches the GPU; and of the plain implementations that
the GPU tests compare with: gradients against differences, codes against their values."""
import ctypes

import numpy as np
import pytest

import adapt_reference as ref


@pytest.fixture(scope="module")
def ev():
    import paper_2605_27390_amd as ev
    return ev


def lora(a=16, b=16, scale=None, n=3, r=16, d_in=64, d_out=32):
    from paper_2605_27390_amd.adapt import _Lora
    return _Lora(a, b, scale, n, r, d_in, d_out)


BAD_SIZES = [dict(n=0), dict(n=65536), dict(r=0), dict(r=12), dict(r=72), dict(d_in=0), dict(d_in=60), dict(d_out=12), dict(d_out=1 << 21),
             dict(d_in=(1 << 20) + 8)]


def test_lora_bytes(ev):
    out = ctypes.c_size_t(0)
    for f in (ev.lib.evospec_lora_backward_workspace_bytes,):
        assert f(ctypes.byref(lora()), 4, 100, ctypes.byref(out)) == 0 and out.value >= 16 * 100 * 4
        for S, T in ((0, 5), (5, 0)):
            assert f(ctypes.byref(lora()), S, T, ctypes.byref(out)) == 0 and out.value == 0
        for bad in BAD_SIZES:
            assert f(ctypes.byref(lora(**bad)), 4, 100, ctypes.byref(out)) == 2, bad
        for S, T in ((-1, 5), (5, -1), ((1 << 16) + 1, 5), (5, 1 << 24)):
            assert f(ctypes.byref(lora()), S, T, ctypes.byref(out)) == 2
        assert f(None, 4, 100, ctypes.byref(out)) == 1 and f(ctypes.byref(lora()), 4, 100, None) == 1
    # past 32 bits
    assert ev.lib.evospec_lora_backward_workspace_bytes(ctypes.byref(lora(r=64)), 1, (1 << 24) - 1, ctypes.byref(out)) == 0 and out.value >= 1 << 32


def test_lora_bytes_of_fewer(ev):
    """A workspace is enough for fewer rows, whatever the requests."""
    for n, r, d in ((1, 8, 64), (1, 32, 4096), (5, 16, 1024), (16, 64, 2048), (300, 32, 4096)):
        before = 0
        for T in (1, 31, 500, 1025, 2049, 9000, 70000):
            out = [ctypes.c_size_t(0) for _ in range(3)]
            for o, S in zip(out, (1, 2, T)):
                assert ev.lib.evospec_lora_backward_workspace_bytes(ctypes.byref(lora(n=n, r=r, d_in=d, d_out=d)), min(S, 1 << 16), T, ctypes.byref(o)) == 0
            assert out[0].value == out[1].value == out[2].value >= before
            before = out[0].value


# Addresses below are never dereferenced: every call that is not an error has nothing to do.
def forward(ev, l=None, x=16, xs=64, off=16, ad=16, S=2, T=5, y=16, ys=32, h=None):
    return ev.lib.evospec_lora_forward(ctypes.byref(l or lora()), x, xs, off, ad, S, T, y, ys, h, None)


def backward(ev, l=None, x=16, xs=64, h=None, dy=16, gs=32, off=16, ad=16, S=2, T=5, dx=None, ds=64, da=16, db=16, ws=16, wb=1 << 30):
    return ev.lib.evospec_lora_backward(ctypes.byref(l or lora()), x, xs, h, dy, gs, off, ad, S, T, dx, ds, da, db, ws, wb, None)


def test_lora_launch_limits(ev):
    out = ctypes.c_size_t(0)
    f = ev.lib.evospec_lora_backward_workspace_bytes
    assert f(ctypes.byref(lora(n=65535, r=64, d_in=4096, d_out=4096)), 1, 5, ctypes.byref(out)) == 2
    assert backward(ev, l=lora(n=65535, r=64, d_in=4096, d_out=4096)) == 2
    assert f(ctypes.byref(lora(n=65535, r=32, d_in=4096, d_out=4160)), 1, 5, ctypes.byref(out)) == 2
    assert f(ctypes.byref(lora(n=65535, r=32, d_in=4096, d_out=2048)), 1, 5, ctypes.byref(out)) == 0


def test_lora_refusals(ev):
    for f in (forward, backward):
        for bad in BAD_SIZES:
            assert f(ev, l=lora(**bad)) == 2, bad
        for bad in (dict(S=-1), dict(T=-1), dict(S=(1 << 16) + 1), dict(T=1 << 24), dict(xs=63), dict(xs=(1 << 26) + 8)):
            assert f(ev, **bad) == 2, bad
        for bad in (dict(x=None), dict(off=None), dict(ad=None), dict(l=lora(a=None)), dict(l=lora(b=None))):
            assert f(ev, **bad) == 1, bad
        for bad in (dict(x=24), dict(xs=68), dict(l=lora(a=8)), dict(l=lora(b=8)), dict(l=lora(scale=2)), dict(h=2)):
            assert f(ev, **bad) == 4, bad
    assert backward(ev, wb=8) == 5 and backward(ev, ws=None) == 1 and backward(ev, ws=8) == 4
    assert forward(ev, ys=24) == 2 and forward(ev, ys=36) == 4 and forward(ev, y=None) == 1 and forward(ev, y=8) == 4
    assert backward(ev, gs=24) == 2 and backward(ev, gs=36) == 4 and backward(ev, dy=None) == 1 and backward(ev, dy=8) == 4
    assert backward(ev, dx=16, ds=56) == 2 and backward(ev, dx=16, ds=68) == 4 and backward(ev, dx=8) == 4
    assert backward(ev, da=None) == 1 and backward(ev, db=None) == 1 and backward(ev, da=8) == 4 and backward(ev, db=8) == 4
    for nothing in (dict(S=0), dict(T=0)):
        assert forward(ev, x=None, y=None, off=None, **nothing) == 0


def kd(ev, h=16, E=3, d=64, W=16, V=100, sup=16, tgt=16, w=None, K=7, T=1.0, type=0, loss=16, dh=16, draft=16, ws=16, wb=1 << 30):
    return ev.lib.evospec_kd_loss(h, E, d, W, V, sup, tgt, w, K, T, type, loss, dh, draft, ws, wb, None)


def test_kd_refusals(ev):
    out = ctypes.c_size_t(0)
    for bad in (dict(E=-1), dict(E=1 << 20), dict(K=0), dict(K=1025), dict(d=0), dict(d=60), dict(d=16392)):
        assert kd(ev, **bad) == 2, bad
        assert ev.lib.evospec_kd_loss_workspace_bytes(bad.get("E", 3), bad.get("K", 7), bad.get("d", 64), ctypes.byref(out)) == 2, bad
    for bad in (dict(V=0), dict(T=0.0), dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan"))):
        assert kd(ev, **bad) == 2, bad
    assert kd(ev, type=1) == 11 and kd(ev, type=3) == 11
    for bad in (dict(h=None), dict(W=None), dict(sup=None), dict(tgt=None), dict(loss=None), dict(dh=None), dict(draft=None)):
        assert kd(ev, **bad) == 1, bad
    for bad in (dict(h=8), dict(W=8), dict(dh=8), dict(ws=8)):
        assert kd(ev, **bad) == 4, bad
    assert ev.lib.evospec_kd_loss_workspace_bytes(1, 256, 64, ctypes.byref(out)) == 0 and out.value > 0
    assert kd(ev, E=1, K=256, wb=out.value - 1) == 5 and kd(ev, E=1, K=256, ws=None) == 1
    assert ev.lib.evospec_kd_loss_workspace_bytes(3, 7, 64, None) == 1
    assert kd(ev, E=0, h=None, W=None, ws=None, wb=0) == 0


def table(ev, *rows):
    from paper_2605_27390_amd.adapt import _Tensor
    return (_Tensor * len(rows))(*[_Tensor(*r) for r in rows])


def step(ev, rows=((16, 16, 5),), count=None, pt=0, gt=0, kind=0, m=16, v=16, scales=8, master=None, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8,
         wd=0.0, t=1, seed=0, schedule=None, gs=None):
    tensors = table(ev, *rows) if rows is not None else None
    return ev.lib.evospec_adamw_step(tensors, len(rows or ()) if count is None else count, pt, gt, kind, m, v, scales, master, lr, b1, b2, eps, wd,
                                     t, seed, schedule, gs, None)


def test_adamw_refusals(ev):
    out = ctypes.c_longlong(0)
    f = ev.lib.evospec_adamw_blocks
    assert f(table(ev, (16, 16, 1), (16, 16, 0), (16, 16, 256), (16, 16, 257)), 4, ctypes.byref(out)) == 0 and out.value == 4
    assert f(None, 0, ctypes.byref(out)) == 0 and out.value == 0
    assert f(None, 1, ctypes.byref(out)) == 1 and f(table(ev, (16, 16, 1)), 1, None) == 1
    assert f(table(ev, (16, 16, -1)), 1, ctypes.byref(out)) == 2 and f(table(ev, (16, 16, (256 << 25) + 1)), 1, ctypes.byref(out)) == 2
    assert step(ev, rows=((16, 16, -1),)) == 2 and step(ev, count=-1) == 2 and step(ev, rows=None, count=2) == 1
    for bad in (dict(pt=3), dict(pt=-1), dict(gt=1), dict(pt=2, gt=0), dict(gt=3), dict(kind=2), dict(kind=-1)):
        assert step(ev, **bad) == 11, bad
    nan, inf = float("nan"), float("inf")
    for bad in (dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=inf), dict(lr=nan), dict(lr=inf),
                dict(wd=nan), dict(t=0), dict(t=-3)):
        assert step(ev, **bad) == 2, bad
    for bad in (dict(m=None), dict(v=None), dict(kind=1, scales=None), dict(rows=((None, 16, 5),)), dict(rows=((16, None, 5),))):
        assert step(ev, **bad) == 1, bad
    for bad in (dict(m=8), dict(v=8), dict(scales=4), dict(master=8), dict(schedule=2), dict(gs=2), dict(rows=((8, 16, 5),)), dict(rows=((16, 24, 5),))):
        assert step(ev, **bad) == 4, bad
    assert step(ev, rows=((None, None, 0),)) == 0 and step(ev, rows=None, count=0) == 0
    g = ev.lib.evospec_adamw_moments
    assert g(16, 16, 8, 3, 1, 16, 16, None) == 11 and g(16, 16, 8, -1, 0, 16, 16, None) == 2 and g(None, 16, 8, 3, 0, 16, 16, None) == 1
    assert g(16, 16, 8, 3, 0, None, 16, None) == 1 and g(16, 16, 4, 3, 0, 16, 16, None) == 4 and g(16, 16, 8, 3, 0, 16, 8, None) == 4
    assert g(None, None, None, 0, 0, None, None, None) == 0


def test_python_refusals(ev):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        ev.LoraBank(x, x)
    with pytest.raises(TypeError):
        ev.kd_loss(x, x, x, x)
    with pytest.raises(TypeError):
        ev.AdamW([x], [x])
    with pytest.raises(ValueError):
        ev.AdamW([x], [x], state="4bit")
    with pytest.raises(ValueError):
        ev.AdamW([], [])


def test_what_overlaps():
    """Rows of one buffer may lie beside each other, and not on one another."""
    import torch
    from paper_2605_27390_amd.adapt import _apart

    def apart(out, x):
        stride = lambda t: t.stride(0) if t.size(0) > 1 else t.size(1)   # noqa: E731
        _apart(out, out.size(0), out.size(1), stride(out), "y", x, x.size(1), stride(x), "x")
    both = torch.zeros(6, 96, dtype=torch.bfloat16)
    x, y = both[:, :64], both[:, 64:]
    apart(y, x)
    apart(x, y)
    apart(both[:2], both[2:4])
    apart(both[:1, :64], both[:1, 64:])
    apart(both[:0], both[:0])
    for a, b in ((x, x), (both[:, :64], both[:, 56:]), (both[:, 56:], both[:, :64]), (both[:3], both[2:5]), (both[:3, :32], both[2:5, 24:56]),
                 (both[:1, :64], both[:1, 56:]), (both.view(12, 48)[:6, :32], both[:, 40:])):
        with pytest.raises(ValueError, match="overlaps"):
            apart(a, b)


# ---------------------------------------------------------------- the plain implementations

def test_lora_gradients_against_differences():
    rng = np.random.default_rng(0)
    T, n, r, d_in, d_out = 9, 3, 8, 16, 24
    x, dy = rng.normal(size=(T, d_in)), rng.normal(size=(T, d_out))
    A, B, scale = rng.normal(size=(n, r, d_in)), rng.normal(size=(n, d_out, r)), rng.normal(size=n)
    off, ad = [1, 4, 4, 6, 8], [2, 0, -1, 2]
    f = lambda x, A, B: np.sum(dy * ref.lora_forward(x, A, B, scale, off, ad, np.zeros((T, d_out)))[0])      # noqa: E731
    dA, _, dB, _, dx, _ = ref.lora_backward(x, dy, A, B, scale, off, ad, np.zeros_like(x))
    args = {"x": x, "A": A, "B": B}
    for name, grad in (("x", dx), ("A", dA), ("B", dB)):
        for at in [tuple(rng.integers(0, k) for k in args[name].shape) for _ in range(25)]:
            up, down = {k: v.copy() for k, v in args.items()}, {k: v.copy() for k, v in args.items()}
            up[name][at] += 1e-3
            down[name][at] -= 1e-3
            # (linear in each: the difference is exact but for roundings)
            assert abs((f(**up) - f(**down)) / 2e-3 - grad[at]) < 1e-9 * (1 + abs(grad[at]))
    assert not dA[1].any() and not dB[0].any() and not dx[0].any() and not dx[4:6].any() and not dx[8:].any()


def test_kd_gradient_against_differences():
    rng = np.random.default_rng(1)
    E, K, d, V, T = 3, 11, 16, 40, 1.7
    h, W = rng.normal(size=(E, d)), rng.normal(size=(V, d)) * 0.5
    support = np.stack([rng.permutation(V)[:K] for _ in range(E)])
    support[1, 4:] = -1
    target, weight = rng.normal(size=(E, K)) * 2, rng.random(E)
    loss, _, dh, _, draft, _ = ref.kd_loss(h, W, support, target, weight, T, 0.0)
    for e in range(E):
        at = support[e] >= 0
        p, q = (np.exp(v[at] / T) / np.sum(np.exp(v[at] / T)) for v in (target[e], draft[e]))
        assert abs(loss[e] - weight[e] * T * T * np.sum(p * np.log(p / q))) < 1e-12
        for i in range(d):
            up, down = h.copy(), h.copy()
            up[e, i] += 1e-4
            down[e, i] -= 1e-4
            diff = (ref.kd_loss(up, W, support, target, weight, T, 0.0)[0] - ref.kd_loss(down, W, support, target, weight, T, 0.0)[0]) / 2e-4
            assert abs(diff[e] - dh[e, i]) < 1e-6 and not np.delete(diff, e).any()


def test_codes():
    """Every code is its value's, whatever the random bits; between two the share of random numbers that go up is the place between them."""
    for values, bias, largest, codes in ((ref.m_values, 7, 448.0, np.arange(127)), (ref.v_values, 15, 61440.0, np.arange(248))):
        y = values(codes)
        assert np.all(np.diff(y) > 0) and y[-1] == largest
        for bits in (0, 1, 40000, 65535):
            assert np.array_equal(ref.grid(y, bits, bias, largest), codes)
        half = (y[1:] + y[:-1]) / 2
        assert np.array_equal(ref.grid(half, 32767, bias, largest), codes[:-1]) and np.array_equal(ref.grid(half, 32768, bias, largest), codes[1:])
    assert ref.scale_for(448.0, 448.0) == 1 and ref.scale_for(448.1, 448.0) == 2 and ref.scale_for(0.0, 448.0) == 2.0 ** -100
    r = ref.random_bits(np.arange(100000), 7, 3)
    for part in (r & 0xffff, r >> 16):                               # (mean of 10^5 of them: standard error 2^16 / sqrt(12 10^5) = 60)
        assert abs(part.mean() - 32767.5) < 300
    assert np.mean(r == ref.random_bits(np.arange(100000), 7, 4)) < 0.01
