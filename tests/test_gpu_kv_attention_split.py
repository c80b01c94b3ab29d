"""Attention whose tokens are shared out over workgroups, and scales of a caller's own: against the formula, within attention_bounds.py."""
import numpy as np
import pytest

import attention_bounds as bounds
import decode_reference as ref
from test_gpu_kv_attention import as_words, random_tree
from test_gpu_kv_cache import i32, to_gpu, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def splits(ev, g, group, S, T, max_rows, max_len):
    """How many workgroups share a row's tokens, from the size of their place."""
    return ev.kv_attention_workspace_bytes(g, group, S, T, max_rows, max_len) // (T * g.heads * group * (g.dim * 4 + 8))


def attend(ev, g, c, q, table, lens, off, type, tree=None, **kw):
    out, lse = ev.kv_attention(q.to(torch_type(type)).cuda(), g, i32(table), i32(lens), i32(off), int(np.diff(off).max()),
                               tree=None if tree is None else as_words(tree), **kw)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


# (dim, kind, type, group, page, lens, rows): up to 128 wavefronts of shares or four at a time, every size of head in both types
@pytest.mark.parametrize("dim,kind,type,group,page,lens,rows", [
    (64, "e4m3", "bf16", 4, 64, [5000, 70, 1], [1, 1, 1]),
    (64, "int8", "fp16", 2, 32, [1700], [1]),
    (96, "e4m3", "fp16", 3, 64, [5000, 31], [1, 1]),
    (96, "int8", "bf16", 1, 128, [1600, 1700], [2, 1]),
    (128, "e4m3", "bf16", 4, 64, [5000, 70, 9], [9, 9, 9]),
    (128, "int8", "fp16", 4, 256, [4100], [1]),
    (128, "e4m3", "fp16", 8, 32, [1999, 64], [5, 3]),
    (192, "e4m3", "bf16", 2, 64, [5000, 1], [1, 1]),
    (192, "int8", "fp16", 1, 32, [1650], [33]),
    (256, "int8", "bf16", 4, 128, [5000, 300], [2, 1]),
    (256, "e4m3", "fp16", 1, 64, [1800], [1]),
])
@pytest.mark.parametrize("tree", [False, True])
def test_every_block_counts_once(ev, dim, kind, type, group, page, lens, rows, tree):
    import torch
    rng = np.random.default_rng(dim + sum(lens))
    S, width = len(lens), (max(lens) + page - 1) // page
    c = ref.Cache(S * width + 2, page, 1, dim, kind, rng)
    table = rng.permutation(c.pages)[:S * width].reshape(S, width)
    bounds.code_by_place(c, table)
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    q = torch.from_numpy(rng.standard_normal((T, group, dim))).to(torch_type(type))
    bits = sum([random_tree(rng, n) for n in rows], []) if tree else None
    g = to_gpu(ev, c)
    assert splits(ev, g, group, S, T, max(rows), max(lens)) > 1
    out, lse = attend(ev, g, c, q, table, lens, off, type, bits, max_len=max(lens))
    want = bounds.attention(c, q.double().numpy(), table, lens, off, group, type, bits)
    assert bounds.differs(out, lse, want) is None


def test_graph_of_a_split_call(ev):
    """Captured once with several workgroups to a row's tokens, and joined: replays follow lengths and queries, other work in between."""
    import torch
    rng = np.random.default_rng(52)
    c = ref.Cache(80, 64, 2, 128, "e4m3", rng)
    g = to_gpu(ev, c)
    table = i32(rng.permutation(80).reshape(2, 40))
    lens, off = i32([2500, 20]), i32([0, 1, 2])
    q = torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    need = ev.kv_attention_workspace_bytes(g, 4, 2, 2, 1, 2560)
    assert splits(ev, g, 4, 2, 2, 1, 2560) > 1
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda: ev.kv_attention(q, g, table, lens, off, 1, max_len=2560, out=out, out_lse=lse, workspace=ws)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a, b in ((2500, 20), (3, 2560), (0, 1), (2560, 2559), (31, 1025)):
        lens.copy_(i32([a, b]))
        q.copy_(torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16))
        ws.fill_(0xFF)                                           # (NaN where nothing is written)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        eager = ev.kv_attention(q, g, table, lens, off, 1, max_len=2560)
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])


@pytest.mark.parametrize("n", [1700, 5000])
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_nan_of_a_share_that_weighs_nothing(ev, n, kind):
    """V has a NaN at a token whose probability is zero in 32 bits, alone in its share of the tokens or not: zero times NaN."""
    import torch
    dim = 64
    k = torch.full((n, 1, dim), -10.0)
    k[5] = 10.0
    v = torch.randn(n, 1, dim, generator=torch.Generator().manual_seed(n))
    v[n - 40, 0, 7] = float("nan")
    q = torch.ones(1, 2, dim, dtype=torch.bfloat16, device="cuda")
    pages = (n + 63) // 64
    at = i32(np.arange(pages)[None])
    c = ev.KVCache(pages, 64, 1, dim, kind)
    ev.kv_write(c, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda(), at, i32([0]), i32([0, n]), n)
    nan = {}
    for max_len in (1, n):                                       # (one workgroup, and several)
        assert (splits(ev, c, 2, 1, 1, 1, max_len) > 1) == (max_len == n)
        out, lse = ev.kv_attention(q, c, at, i32([n]), i32([0, 1]), 1, max_len=max_len)
        assert torch.isfinite(lse).all()
        nan[max_len] = torch.isnan(out)
    want = torch.zeros(1, 2, dim, dtype=torch.bool, device="cuda")
    want[..., 7] = True
    assert torch.equal(nan[1], want) and torch.equal(nan[n], want)


@pytest.mark.parametrize("kind,type", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("zero", [0.0, -0.0, 2.0 ** -140])
def test_scales_of_zero(ev, kind, type, zero):
    """A caller's own scales: those of V and of K that are zero, or next to it, make values of zero, whatever the codes are."""
    import torch
    rng = np.random.default_rng(50)
    dim, page, lens, rows = 64, 64, [300, 40], [3, 1]
    for part in (0, 1, 2):                                       # K, V, both
        for share in (0.3, 1.0):
            c = ref.Cache(12, page, 2, dim, kind, rng)
            table = rng.permutation(12)[:10].reshape(2, 5)
            w = [part] if part < 2 else [0, 1]
            for i in w:
                c.scales[..., i][rng.random(c.scales[..., i].shape) < share] = zero
            q = torch.from_numpy(rng.standard_normal((4, 4, dim))).to(torch_type(type))
            off = [0, 3, 4]
            out, lse = attend(ev, to_gpu(ev, c), c, q, table, lens, off, type)
            want = bounds.attention(c, q.double().numpy(), table, lens, off, 2, type)
            assert bounds.differs(out, lse, want) is None, (part, share)
            if part and share == 1.0:
                assert (out == 0).all()
