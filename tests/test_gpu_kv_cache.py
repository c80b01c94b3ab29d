"""The 8-bit cache on the GPU against its definition: bytes and scales are equal, values read back are rounded once."""
import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "fp16", "fp32"]


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def torch_type(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def to_gpu(ev, c):
    import torch
    return ev.KVCache(c.pages, c.page, c.heads, c.dim, c.kind, data=torch.from_numpy(c.data.copy()).cuda(),
                      scales=torch.from_numpy(c.scales.copy()).cuda())


def same(g, c):
    """Bytes and scales of a GPU cache are the host's (a NaN code may carry a sign)."""
    data, scales = g.data.cpu().numpy(), g.scales.cpu().numpy()
    if c.kind == "e4m3":
        data, want = np.where(data == 255, 127, data), np.where(c.data == 255, 127, c.data)
    else:
        want = c.data
    assert np.array_equal(scales.view(np.uint32), c.scales.view(np.uint32))
    assert np.array_equal(data, want)


def new_rows(rng, T, heads, dim, type, spread=3.0, stride=None):
    """(k, v on the GPU, k, v as float32 on the host) of magnitudes that differ between rows; rows `stride` elements apart."""
    import torch
    out = []
    for _ in range(2):
        x = rng.standard_normal((T, heads, dim)) * 2.0 ** rng.uniform(-spread, spread, (T, heads, 1))
        t = torch.from_numpy(x).to(torch_type(type))
        g = t.cuda()
        if stride:
            wide = torch.full((T, stride), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, :heads * dim] = g.view(T, -1)
            g = wide[:, :heads * dim].view(T, heads, dim)
        out.append((g, t.float().numpy()))
    return out[0][0], out[1][0], out[0][1], out[1][1]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dim,heads,page,type,starts,rows", [
    (64, 2, 32, "bf16", [0], [1]),                              # one token
    (64, 1, 32, "fp32", [31, 32, 33], [1, 1, 1]),               # around the border of a block
    (96, 3, 64, "fp16", [0, 40, 7], [64, 33, 0]),               # ragged, one sequence without rows
    (128, 2, 128, "bf16", [5, 0, 100, 64], [60, 129, 2, 32]),
    (192, 1, 64, "fp32", [63, 20], [70, 5]),
    (256, 2, 256, "fp16", [250, 0], [10, 31]),
])
def test_write(ev, kind, dim, heads, page, type, starts, rows):
    import torch
    rng = np.random.default_rng(dim + sum(rows))
    S = len(starts)
    width = max((a + n + page - 1) // page for a, n in zip(starts, rows)) + 1
    c = ref.Cache(S * width + 2, page, heads, dim, kind, rng)
    table = rng.permutation(c.pages)[:S * width].reshape(S, width)
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    gk, gv, k, v = new_rows(rng, T, heads, dim, type)
    g = to_gpu(ev, c)
    ev.kv_write(g, gk, gv, i32(table), i32(starts), i32(off), max(rows))
    before = c.data.copy()
    c.write(k, v, table, starts, off)
    # what a block holds behind its last token is not specified: compared are the others, and blocks that are not touched
    for s in range(S):
        end = starts[s] + rows[s]
        if rows[s] and end % 32:
            p, b = c.place(table, s, end // 32)
            for h in range(heads):
                gk_, gv_ = ref.block_codes(g.data[p, h, b].cpu().numpy())
                wk, wv = ref.block_codes(c.data[p, h, b])
                wk, wv = wk.copy(), wv.copy()
                wk[end % 32:], wv[end % 32:] = gk_[end % 32:], gv_[end % 32:]
                c.data[p, h, b] = ref.block_bytes(wk, wv)
    same(g, c)
    assert (c.data != before).any()
    # and back, in every type
    for back in TYPES:
        n = int(off[-1])
        ok, ov = ev.kv_read(g, i32(table), i32(starts), i32(off), max(rows), n, torch_type(back))
        for s in range(S):
            wk, wv, there = c.values(table, s, starts[s] + rows[s])
            assert there.all()
            for got, want in ((ok, wk), (ov, wv)):
                want = torch.from_numpy(want[starts[s]:].astype(np.float32)).to(torch_type(back))
                assert torch.equal(got[off[s]:off[s + 1]].cpu(), want), (s, back)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_token_by_token(ev, kind):
    """A block filled by single tokens of growing magnitudes: its codes are rescaled on the way."""
    rng = np.random.default_rng(3)
    c = ref.Cache(3, 32, 1, 64, kind, rng)
    table, g = np.array([[2, 0]]), to_gpu(ev, c)
    for t in range(40):
        gk, gv, k, v = new_rows(rng, 1, 1, 64, "bf16", spread=1.0 + t / 4)
        ev.kv_write(g, gk, gv, i32(table), i32([t]), i32([0, 1]), 1)
        c.write(k, v, table, [t], [0, 1])
        ok, ov = ev.kv_read(g, i32(table), i32([0]), i32([0, t + 1]), t + 1, t + 1, torch_type("fp32"))
        wk, wv, _ = c.values(table, 0, t + 1)
        assert np.array_equal(ok.cpu().numpy(), wk.astype(np.float32)) and np.array_equal(ov.cpu().numpy(), wv.astype(np.float32)), t


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("type", TYPES)
def test_special_values(ev, kind, type):
    """NaN stays NaN and is flagged, infinities saturate, zeros and the smallest and largest magnitudes keep."""
    import torch
    rng = np.random.default_rng(5)
    T, heads, dim = 128, 2, 64
    x = rng.standard_normal((2, T, heads, dim))
    t = torch.from_numpy(x).to(torch_type(type))
    t[0, 3, 0, 5] = float("nan")
    t[1, 40, 1, 6] = float("inf")
    t[0, 41, 1, 7] = float("-inf")
    t[1, 33, 0, 0] = float("nan")
    t[:, 64:96, 0] = 0                                          # a block of zeros
    t[0, 70, 1] = torch.finfo(t.dtype).max
    t[1, 70, 1, :9] = -torch.finfo(t.dtype).max
    t[0, 96:128, 0] = torch.finfo(t.dtype).tiny                # all of a block at the smallest normal
    t[0, 96:128, 1] = float("nan")                              # nothing but NaN
    c = ref.Cache(2, 64, heads, dim, kind)
    table = np.array([[1, 0]])
    g = to_gpu(ev, c)
    d = t.cuda()
    ev.kv_write(g, d[0], d[1], i32(table), i32([0]), i32([0, T]), T)
    f = t.float().numpy()
    c.write(f[0], f[1], table, [0], [0, T])
    same(g, c)
    assert np.signbit(c.scales).sum() == 3 and np.isfinite(c.scales).all()


def test_rows_of_a_fused_projection_and_another_stream(ev):
    """K and V beside each other in wider rows, on a stream of their own."""
    import torch
    rng = np.random.default_rng(6)
    T, heads, dim = 75, 2, 128
    c = ref.Cache(4, 64, heads, dim, "e4m3", rng)
    table, g = np.array([[3, 1]]), to_gpu(ev, c)
    gk, gv, k, v = new_rows(rng, T, heads, dim, "bf16", stride=heads * dim * 2 + 40)
    at, off, start = i32(table), i32([0, T]), i32([0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ev.kv_write(g, gk, gv, at, start, off, T)
        ok, ov = ev.kv_read(g, at, start, off, T, T, torch.float32)
    side.synchronize()
    c.write(k, v, table, [0], [0, T])
    wk, wv, _ = c.values(table, 0, T)
    assert np.array_equal(ok.cpu().numpy(), wk.astype(np.float32)) and np.array_equal(ov.cpu().numpy(), wv.astype(np.float32))


def test_pages_that_are_not_there(ev):
    """Entries out of range, and tokens past the table: not written, read back as zeros; neighbours are untouched."""
    rng = np.random.default_rng(7)
    T, heads, dim = 200, 1, 64
    c = ref.Cache(3, 64, heads, dim, "int8", rng)
    table = np.array([[0, -1, 2]])                              # 192 tokens of 200, 64 of them nowhere
    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        table[0, 1] = bad
        g = to_gpu(ev, c)
        gk, gv, k, v = new_rows(rng, T, heads, dim, "fp32")
        ev.kv_write(g, gk, gv, i32(table), i32([0]), i32([0, T]), T)
        want = ref.Cache(3, 64, heads, dim, "int8", rng)
        want.data, want.scales = c.data.copy(), c.scales.copy()
        want.write(k, v, table, [0], [0, T])
        same(g, want)
        assert np.array_equal(want.data[1], c.data[1])
        ok, ov = ev.kv_read(g, i32(table), i32([0]), i32([0, T]), T, T, torch_type("fp32"))
        wk, wv, there = want.values(table, 0, T)
        assert there.sum() == 128 and np.array_equal(ok.cpu().numpy(), wk.astype(np.float32)) and np.array_equal(ov.cpu().numpy(), wv.astype(np.float32))


def test_offsets_that_do_not_hold(ev):
    """row_off past the rows, falling, or more rows than max_rows: no more than what there is is touched."""
    import torch
    rng = np.random.default_rng(8)
    heads, dim = 1, 64
    c = ref.Cache(4, 32, heads, dim, "e4m3", rng)
    table = np.array([[0, 1], [2, 3]])
    gk, gv, k, v = new_rows(rng, 20, heads, dim, "bf16")
    for off, starts, most, does in (([0, 10, 1000], [0, 0], 20, [0, 10, 20]), ([0, 15, 5], [0, 0], 20, [0, 15, 15]),
                                    ([-7, 10, 20], [0, 0], 20, [0, 10, 20]), ([0, 10, 20], [-5, 0], 20, [0, 10, 20])):
        g, want = to_gpu(ev, c), ref.Cache(4, 32, heads, dim, "e4m3", rng)
        want.data, want.scales = c.data.copy(), c.scales.copy()
        ev.kv_write(g, gk, gv, i32(table), i32(starts), i32(off), most)
        want.write(k, v, table, [0, 0], does)
        for s in range(2):
            n = does[s + 1] - does[s]
            if n:
                got = ev.kv_read(g, i32(table[s:s + 1]), i32([0]), i32([0, n]), n, n, torch.float32)
                for a, b in zip(got, want.values(table, s, n)):
                    assert np.array_equal(a.cpu().numpy(), b)
            else:
                assert np.array_equal(g.data[table[s]].cpu().numpy(), c.data[table[s]])
    # rows past max_rows
    g = to_gpu(ev, c)
    ev.kv_write(g, gk, gv, i32(table[:1]), i32([0]), i32([0, 20]), 8)
    ok, _ = ev.kv_read(g, i32(table[:1]), i32([0]), i32([0, 8]), 8, 8, torch.float32)
    want = ref.Cache(4, 32, heads, dim, "e4m3", rng)
    want.write(k[:8], v[:8], table[:1], [0], [0, 8])
    assert np.array_equal(ok.cpu().numpy(), want.values(table, 0, 8)[0])


def test_wrapper_refusals(ev):
    import torch
    c = ev.KVCache(4, 32, 2, 64)
    t, s, o = i32([[0, 1]]), i32([0]), i32([0, 3])
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(k=k[:, :1]), dict(k=k.float()), dict(v=k[:2]), dict(k=k.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(k=k.cpu()), dict(table=i32([0, 1])), dict(starts=i32([0, 1])), dict(off=i32([0])), dict(table=i32([[0, 1]]).long())):
        with pytest.raises((TypeError, ValueError)):
            ev.kv_write(c, bad.get("k", k), bad.get("v", k), bad.get("table", t), bad.get("starts", s), bad.get("off", o), 3)
    with pytest.raises(ev.EvospecError) as e:                  # rows that start between 16-byte borders
        wide = torch.zeros(3, 132, dtype=torch.bfloat16, device="cuda")[:, :128].view(3, 2, 64)
        ev.kv_write(c, wide, wide, t, s, o, 3)
    assert e.value.status == 4
    with pytest.raises(TypeError):
        ev.kv_read(c, t, s, o, 3, 3, torch.int8)
    with pytest.raises(ValueError):
        ev.kv_read(c, t, s, o, 3, 3, out_k=torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        ev.KVCache(4, 32, 2, 64, data=torch.zeros(100, dtype=torch.uint8, device="cuda"))


def test_offsets_past_32_bits(ev):
    """Pages behind the first 4 GiB of a cache."""
    import torch
    rng = np.random.default_rng(9)
    heads, dim, page = 8, 256, 256
    pages = 4500                                               # of 1 MiB
    g = ev.KVCache(pages, page, heads, dim, "e4m3")
    T = 40
    gk, gv, k, v = new_rows(rng, T, heads, dim, "bf16")
    table = np.array([[pages - 1]])
    ev.kv_write(g, gk, gv, i32(table), i32([0]), i32([0, T]), T)
    ok, ov = ev.kv_read(g, i32(table), i32([0]), i32([0, T]), T, T, torch.float32)
    want = ref.Cache(1, page, heads, dim, "e4m3")
    want.write(k, v, np.array([[0]]), [0], [0, T])
    wk, wv, _ = want.values(np.array([[0]]), 0, T)
    assert np.array_equal(ok.cpu().numpy(), wk.astype(np.float32)) and np.array_equal(ov.cpu().numpy(), wv.astype(np.float32))
