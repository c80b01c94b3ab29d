"""Host-only checks of include/evospec_decode.h: sizes, and refusals before anything touches the GPU; and of the plain
implementations that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

import decode_reference as ref


@pytest.fixture(scope="module")
def ev():
    import paper_2605_27390_amd as ev
    return ev


def cache(ev, pages=4, page=64, heads=2, dim=128, kind=0, data=16, scales=16):
    from paper_2605_27390_amd.decode import _Cache
    return _Cache(data, scales, pages, page, heads, dim, kind)


BAD_CACHES = [(dict(kind=2), 11), (dict(kind=-1), 11), (dict(pages=0), 2), (dict(heads=0), 2), (dict(page=16), 2),
              (dict(page=96), 2), (dict(page=512), 2), (dict(dim=32), 2), (dict(dim=80), 2), (dict(dim=512), 2)]


def test_cache_bytes(ev):
    d, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
    f = ev.lib.evospec_kv_cache_bytes
    assert f(ctypes.byref(cache(ev)), ctypes.byref(d), ctypes.byref(s)) == 0
    assert d.value == 4 * 2 * 64 * 128 * 2 and s.value == 4 * 2 * 2 * 2 * 4
    # past 32 bits
    assert f(ctypes.byref(cache(ev, pages=1 << 20, page=256, heads=8)), ctypes.byref(d), ctypes.byref(s)) == 0
    assert d.value == (1 << 20) * 256 * 8 * 128 * 2
    for bad, status in BAD_CACHES:
        assert f(ctypes.byref(cache(ev, **bad)), ctypes.byref(d), ctypes.byref(s)) == status, bad
    assert f(None, ctypes.byref(d), ctypes.byref(s)) == 1
    assert f(ctypes.byref(cache(ev)), None, ctypes.byref(s)) == 1


# Addresses below are never dereferenced: every call that is not an error has nothing to do.
def write(ev, c=None, k=16, ks=256, v=16, vs=256, type=0, T=5, table=16, width=3, starts=16, off=16, S=2, most=4):
    return ev.lib.evospec_kv_write(ctypes.byref(c or cache(ev)), k, ks, v, vs, type, T, table, width, starts, off, S, most, None)


def test_write_refusals(ev):
    for bad, status in BAD_CACHES:
        assert write(ev, c=cache(ev, **bad)) == status, bad
    assert write(ev, type=3) == 11 and write(ev, type=-1) == 11
    for bad in (dict(T=-1), dict(width=0), dict(S=-1), dict(most=-1), dict(ks=255), dict(vs=128), dict(most=1 << 29)):
        assert write(ev, **bad) == 2, bad
    assert write(ev, ks=257) == 4 and write(ev, vs=260) == 4 and write(ev, type=2, ks=258) == 4
    assert write(ev, S=1 << 24, most=1 << 20) == 2                       # more workgroups than a launch takes
    for bad in (dict(k=None), dict(v=None), dict(table=None), dict(starts=None), dict(off=None), dict(c=cache(ev, data=None)),
                dict(c=cache(ev, scales=None))):
        assert write(ev, **bad) == 1, bad
    for bad in (dict(k=8), dict(v=24), dict(c=cache(ev, data=8)), dict(c=cache(ev, scales=4))):
        assert write(ev, **bad) == 4, bad
    for nothing in (dict(T=0), dict(S=0), dict(most=0)):
        assert write(ev, k=None, **nothing) == 0, nothing


def read(ev, c=None, table=16, width=3, starts=16, off=16, S=2, most=4, T=5, type=0, k=16, v=16):
    return ev.lib.evospec_kv_read(ctypes.byref(c or cache(ev)), table, width, starts, off, S, most, T, type, k, v, None)


def test_read_refusals(ev):
    for bad, status in BAD_CACHES:
        assert read(ev, c=cache(ev, **bad)) == status, bad
    assert read(ev, type=3) == 11
    for bad in (dict(T=-1), dict(width=0), dict(S=-1), dict(most=-1)):
        assert read(ev, **bad) == 2, bad
    for bad in (dict(k=None), dict(v=None), dict(table=None), dict(starts=None), dict(off=None), dict(c=cache(ev, data=None))):
        assert read(ev, **bad) == 1, bad
    assert read(ev, k=8) == 4 and read(ev, v=8) == 4
    assert read(ev, T=0, k=None) == 0 and read(ev, S=0, k=None) == 0 and read(ev, most=0, k=None) == 0


def attend(ev, c=None, q=16, qs=1024, type=0, T=5, group=4, table=16, width=3, lens=16, off=16, S=2, most=4, max_len=192, tree=None,
           scale=0.1, out=16, lse=16, ws=16, nws=1 << 40):
    return ev.lib.evospec_kv_attention(ctypes.byref(c or cache(ev)), q, qs, type, T, group, table, width, lens, off, S, most, max_len,
                                       tree, scale, out, lse, ws, nws, None)


def test_attention_refusals(ev):
    for bad, status in BAD_CACHES:
        assert attend(ev, c=cache(ev, **bad)) == status, bad
    assert attend(ev, type=2) == 11 and attend(ev, type=-1) == 11
    for bad in (dict(T=-1), dict(width=0), dict(S=-1), dict(most=-1), dict(group=0), dict(max_len=-1), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan")), dict(qs=1023), dict(tree=16, most=65),
                dict(group=1024, most=1 << 27), dict(group=1024, T=1 << 21)):
        assert attend(ev, **bad) == 2, bad
    assert attend(ev, qs=1028) == 4
    for bad in (dict(q=None), dict(table=None), dict(lens=None), dict(off=None), dict(out=None), dict(c=cache(ev, data=None))):
        assert attend(ev, **bad) == 1, bad
    assert attend(ev, q=8) == 4 and attend(ev, out=8) == 4 and attend(ev, ws=8) == 4
    assert attend(ev, T=0, q=None) == 0 and attend(ev, S=0, q=None) == 0 and attend(ev, most=0, q=None) == 0
    # a long sequence is split, and the parts need a place
    n = ctypes.c_size_t(0)
    w = ev.lib.evospec_kv_attention_workspace_bytes
    assert w(ctypes.byref(cache(ev)), 4, 1, 1, 1, 100000, ctypes.byref(n)) == 0 and n.value > 0
    assert attend(ev, S=1, T=1, most=1, max_len=100000, nws=n.value - 1) == 5
    assert attend(ev, S=1, T=1, most=1, max_len=100000, ws=None) == 1
    assert w(ctypes.byref(cache(ev)), 4, 1, 1, 1, 100000, None) == 1
    assert w(ctypes.byref(cache(ev)), 0, 1, 1, 1, 100000, ctypes.byref(n)) == 2
    assert w(ctypes.byref(cache(ev)), 4, 0, 0, 0, 0, ctypes.byref(n)) == 0 and n.value == 0


def draw(ev, z=16, stride=100, type=2, M=3, V=100, u=16, out=16, lp=16, ws=16, nws=1 << 40):
    return ev.lib.evospec_sample(z, stride, type, M, V, u, None, None, None, None, None, out, lp, ws, nws, None)


def test_sample_refusals(ev):
    assert draw(ev, type=3) == 11 and draw(ev, type=-1) == 11
    for bad in (dict(M=-1), dict(V=0), dict(V=(1 << 20) + 1, stride=1 << 21), dict(stride=99)):
        assert draw(ev, **bad) == 2, bad
    for bad in (dict(z=None), dict(u=None), dict(out=None)):
        assert draw(ev, **bad) == 1, bad
    assert draw(ev, z=18) == 4 and draw(ev, z=17, type=0) == 4 and draw(ev, ws=8) == 4
    assert draw(ev, M=0, z=None) == 0
    n = ctypes.c_size_t(0)
    w = ev.lib.evospec_sample_workspace_bytes
    assert w(3, 100, ctypes.byref(n)) == 0
    if n.value:
        assert draw(ev, nws=n.value - 1) == 5 and draw(ev, ws=None) == 1
    assert w(3, 100, None) == 1 and w(-1, 100, ctypes.byref(n)) == 2 and w(3, 0, ctypes.byref(n)) == 2


def test_more_threads_than_a_launch_takes(ev):
    """2^32 threads of a launch and more are refused here."""
    c = cache(ev, heads=4)
    assert write(ev, c=c, S=1 << 22, most=1, ks=512, vs=512) == 2 and read(ev, c=c, S=1 << 22, most=1) == 2
    assert attend(ev, c=c, S=1 << 22, most=1, qs=2048) == 2 and attend(ev, T=1 << 21, most=1, max_len=1 << 20, S=1) == 2
    n = ctypes.c_size_t(0)
    w = ev.lib.evospec_sample_workspace_bytes
    assert draw(ev, M=1 << 22) == 2 and w(1 << 22, 100, ctypes.byref(n)) == 2 and w((1 << 22) - 1, 100, ctypes.byref(n)) == 0
    assert w(1 << 21, 20481, ctypes.byref(n)) == 2 and w(1 << 21, 20480, ctypes.byref(n)) == 0
    # what is just below is not (the null pointer is what it stops at)
    assert write(ev, c=c, S=(1 << 22) - 256, most=1, ks=512, vs=512, k=None) == 1
    assert attend(ev, c=c, S=(1 << 22) - 256, most=1, qs=2048, q=None) == 1


def test_sample_workspace_of_fewer_rows(ev):
    """Scratch for M rows is enough for fewer."""
    for V in (1, 4096, 20480, 20481, 50000, 151936, 1 << 20):
        sizes = [ev.sample_workspace_bytes(M, V) for M in list(range(0, 300)) + [511, 512, 513, 960]]
        assert sizes == sorted(sizes) and sizes[0] == 0


def test_wrapper_refusals_need_no_gpu(ev):
    import torch
    with pytest.raises(ValueError):
        ev.KVCache(4, 64, 2, 128, kind="int4")
    with pytest.raises(ev.EvospecError) as e:
        ev.KVCache(4, 48, 2, 128)
    assert e.value.status == 2
    with pytest.raises(TypeError):
        ev.sample(torch.zeros(2, 10), torch.zeros(2))


# ---------------------------------------------------------------- the plain implementations themselves

def test_reference_codes():
    v = ref.E4M3
    assert v[0x7e] == 448 and v[0xfe] == -448 and np.isnan(v[0x7f]) and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6
    codes = np.arange(256, dtype=np.uint8)
    back = ref.encode(v, "e4m3")
    assert np.array_equal(back[np.isfinite(v)], codes[np.isfinite(v)])
    # halfway between neighbours: to the even mantissa; past the largest: saturated
    mid = (v[8:126] + v[9:127]) / 2
    assert np.all(ref.encode(mid, "e4m3") % 2 == 0)
    assert ref.encode([1e9, -1e9, np.inf, np.nan], "e4m3").tolist() == [126, 254, 126, 127]
    assert ref.encode([126.5, -127.6, np.nan, 0.5, 1.5], "int8").tolist() == [126, 129, 128, 0, 2]


def test_reference_layout_is_a_permutation():
    rng = np.random.default_rng(0)
    k, v = rng.integers(0, 256, (2, 32, 96), dtype=np.uint8)
    b = ref.block_bytes(k, v)
    bk, bv = ref.block_codes(b)
    assert np.array_equal(bk, k) and np.array_equal(bv, v)
    # token 21 = 8 * 2 + 4 * 1 + 1, dimension 70 = 2 * 32 + 6
    assert b[0][2 * 1024 + 0 * 512 + 21 * 16 + 6] == k[21, 70]
    assert b[1][2 * 1024 + 1 * 512 + 6 * 16 + 4 * 2 + 1] == v[21, 70]


def test_reference_scale():
    assert ref.scale_of(448.0, "e4m3") == 1 and ref.scale_of(448.5, "e4m3") == 2 and ref.scale_of(224.0, "e4m3") == 0.5
    assert ref.scale_of(0.0, "e4m3") == 2.0 ** -100 and ref.scale_of(254.0, "int8") == 2 and ref.scale_of(0.0, "int8") == np.float32(2.0 ** -100)


def test_reference_sample_by_hand():
    z = np.log(np.array([[0.1, 0.4, 0.2, 0.3]]))
    pick = lambda u, **kw: int(ref.sample(z, [u], **kw)[0][0])            # noqa: E731
    assert [pick(u) for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]
    assert pick(0.99, top_k=[2]) == 3 and pick(0.99, top_p=[0.75]) == 2 and pick(0.99, min_p=[0.6]) == 3
    assert pick(0.99, temperature=[0.0]) == 1 and pick(0.99, top_p=[0.0]) == 1
    assert pick(0.0, ids=[9, 8, 7, 6]) == 8
    assert ref.sample(np.full((1, 4), -np.inf), [0.5])[0][0] == -1
