"""Attention over the 8-bit cache on the GPU against the formula in 64 bits.

Tolerances.  Codes times scales and products with q are exact in what the matrix cores take; a score is a sum of dim products in
32 bits, off by at most E = (dim + 8) 2^-24 sum |q k| scale, which moves every probability by a factor of 1 +- 2 E at most (its own
and the normaliser's); the exponential and its argument add 2^-20.  Probabilities are rounded to fp16 (2^-11 of each, or 2^-25 of
the reference where they are below its 2^-14), the output to its type.  With A = sum softmax |v|, n tokens and v_max the
largest |v| times the ratio of the scales:
    |out - exact| <= |exact| eps / 2 + A (2^-11 + 2 E + 2^-20 + n 2^-24) + n 2^-25 v_max,    |lse - exact| <= E + 2^-20 (1 + |lse|)."""
import numpy as np
import pytest

import decode_reference as ref
from test_gpu_kv_cache import i32, to_gpu, torch_type

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ev():
    import torch
    assert torch.cuda.is_available()
    import paper_2605_27390_amd as ev
    return ev


def random_tree(rng, n):
    """Bits of a tree of n nodes: each sees its ancestors and itself."""
    bits = []
    for j in range(n):
        bits.append((bits[int(rng.integers(0, j))] if j else 0) | 1 << j)
    return bits


def as_words(bits):
    import torch
    return torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device="cuda")


def check(got, lse, c, want, want_lse, weight, score, v_max, n, type):
    import torch
    eps = torch.finfo(torch_type(type)).eps
    E = ((c.dim + 8) * 2.0 ** -24 * score)
    tol = np.abs(want) * eps / 2 + weight * (2.0 ** -11 + 2 * E + 2.0 ** -20 + n * 2.0 ** -24)[..., None] + n * 2.0 ** -25 * v_max
    off = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (off <= tol).all(), (np.unravel_index((off - tol).argmax(), off.shape), (off / tol).max())
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(lse), empty) and (got[empty] == 0).all()
    lse, want_lse = lse[~empty], want_lse[~empty]
    assert (np.abs(lse - want_lse) <= E[~empty] + 2.0 ** -20 * (1 + np.abs(want_lse))).all()


def case(ev, seed, kind, type, dim, heads, group, page, lens, rows, tree=False, scale=None, q_scale=1.0, stride=None, max_len=None,
         extra_width=0, trees=None):
    import torch
    rng = np.random.default_rng(seed)
    S = len(lens)
    width = max(1, max((n + page - 1) // page for n in lens)) + extra_width
    c = ref.Cache(S * width + 2, page, heads, dim, kind, rng)
    table = rng.permutation(c.pages)[:S * width].reshape(S, width)
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    q = (torch.from_numpy(rng.standard_normal((T, heads * group, dim))) * q_scale).to(torch_type(type))
    g = q.cuda()
    if stride:
        wide = torch.full((T, stride), float("nan"), dtype=q.dtype, device="cuda")
        wide[:, :heads * group * dim] = g.view(T, -1)
        g = wide[:, :heads * group * dim].view(T, heads * group, dim)
    bits = None
    if tree:
        bits = trees if trees is not None else sum([random_tree(rng, n) for n in rows], [])
    gc = to_gpu(ev, c)
    out, lse = ev.kv_attention(g, gc, i32(table), i32(lens), i32(off), max(rows), max_len=max_len, tree=as_words(bits) if tree else None,
                               scale=scale)
    want = ref.attention(c, q.double().numpy(), table, lens, off, group, bits, dim ** -0.5 if scale is None else scale)
    s = np.abs(c.scales[..., 1].astype(np.float64))
    v_max = np.nanmax(np.abs(ref.decode(c.data[:, :, :, 1], kind)) * s[..., None]) * (s.max() / s.min())
    check(out.double().cpu().numpy(), lse.double().cpu().numpy(), c, *want, v_max, max(1, max(lens)), type)
    return out, lse


@pytest.mark.parametrize("kind,type", [("e4m3", "bf16"), ("e4m3", "fp16"), ("int8", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("dim,heads,group,page,lens", [
    (64, 2, 4, 32, [1]),                                        # a first token
    (64, 1, 1, 32, [31, 32, 33]),                               # around a block
    (96, 2, 3, 64, [100, 1, 65]),
    (128, 2, 4, 64, [700, 0, 5]),                               # a sequence without tokens: its row sees nothing
    (192, 1, 7, 128, [400]),
    (256, 1, 8, 256, [300, 257]),
])
def test_single_tokens(ev, kind, type, dim, heads, group, page, lens):
    case(ev, dim + len(lens), kind, type, dim, heads, group, page, lens, [1] * len(lens))


@pytest.mark.parametrize("kind,type", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("dim,heads,group,page,lens,rows", [
    (128, 2, 4, 64, [300, 61], [60, 60]),                       # 240 rows of a head
    (64, 1, 4, 32, [64, 100], [64, 3]),                         # all 64 bits
    (128, 1, 8, 32, [90], [7]),                                 # 56 rows
    (96, 1, 1, 64, [45, 20, 33], [12, 20, 1]),                  # no context before the tree
    (256, 1, 4, 64, [80], [20]),
    (192, 2, 2, 128, [200], [30]),
])
def test_trees(ev, kind, type, dim, heads, group, page, lens, rows):
    case(ev, dim + sum(rows), kind, type, dim, heads, group, page, lens, rows, tree=True)


@pytest.mark.parametrize("kind,type", [("e4m3", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("dim,heads,group,page,lens,rows", [
    (128, 1, 4, 64, [200], [100]),                              # several workgroups of rows
    (64, 2, 1, 32, [40, 129, 33], [40, 70, 2]),
    (128, 1, 2, 256, [300], [300]),
    (256, 1, 2, 64, [70], [33]),
    (96, 1, 5, 64, [77], [50]),
    (192, 1, 1, 32, [130], [130]),
])
def test_chunks(ev, kind, type, dim, heads, group, page, lens, rows):
    case(ev, dim + sum(rows), kind, type, dim, heads, group, page, lens, rows)


@pytest.mark.parametrize("kind,type,dim", [("e4m3", "bf16", 64), ("int8", "fp16", 64), ("e4m3", "fp16", 96), ("int8", "bf16", 128)])
@pytest.mark.parametrize("tree", [False, True])
def test_many_rows(ev, kind, type, dim, tree):
    """Enough rows of enough heads that a wavefront takes two tiles of them; the last tile is ragged, some sequences are short."""
    rows = [33 + (5 * i) % 32 for i in range(32)]
    rows[3], rows[7], rows[31] = 64, 1, 40
    lens = [r + (7 * i) % 50 for i, r in enumerate(rows)]
    case(ev, dim, kind, type, dim, 16, 1, 32, lens, rows, tree=tree)


def test_nan_with_many_rows(ev):
    """As below, where a wavefront has two tiles: a NaN in V of one node of one sequence."""
    import torch
    rng = np.random.default_rng(42)
    S, n, ctx, heads, dim = 32, 40, 30, 16, 64
    width = 3
    kv = torch.from_numpy(rng.standard_normal((2, S * (ctx + n), heads, dim))).to(torch.bfloat16).cuda()
    q = torch.from_numpy(rng.standard_normal((S * n, heads, dim))).to(torch.bfloat16).cuda()
    bits = sum([random_tree(rng, n) for _ in range(S)], [])
    at, zero = i32(np.arange(S * width).reshape(S, width)), i32([0] * S)
    off, whole = i32(np.arange(S + 1) * n), i32(np.arange(S + 1) * (ctx + n))
    s, node, h = 5, 17, 9
    got = []
    for bad in (False, True):
        x = kv.clone()
        if bad:
            x[1, s * (ctx + n) + ctx + node, h, 50] = float("nan")
        c = ev.KVCache(S * width, 32, heads, dim)
        ev.kv_write(c, x[0], x[1], at, zero, whole, ctx + n)
        got.append(ev.kv_attention(q, c, at, i32([ctx + n] * S), off, n, tree=as_words(bits)))
    nan = torch.isnan(got[1][0])
    sees = [s * n + j for j in range(n) if bits[s * n + j] >> node & 1]
    want = torch.zeros_like(nan)
    want[sees, h, 50] = True
    assert sees and torch.equal(nan, want)
    assert torch.equal(got[0][0][~want], got[1][0][~want]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("rows", [1, 9, 17, 33])
def test_split_over_long_sequences(ev, rows):
    """Long and short sequences in one call: several workgroups share the tokens of a row, some of them find none."""
    case(ev, 20 + rows, "e4m3", "bf16", 128, 1, 4, 64, [5000, 70, rows], [rows] * 3)


def test_rows_that_see_nothing(ev):
    """Tree words of zero without a context; more rows than tokens."""
    case(ev, 30, "e4m3", "bf16", 64, 1, 2, 32, [5, 40], [5, 4], tree=True, trees=[1, 0, 4, 0, 16, 0, 1, 2, 0])
    case(ev, 31, "int8", "bf16", 64, 1, 2, 32, [3, 0], [5, 2])


def test_large_scores_and_scale(ev):
    """Softmax that one token takes, and scores far below and above zero."""
    case(ev, 32, "int8", "bf16", 128, 1, 4, 64, [500], [3], q_scale=40.0)
    case(ev, 33, "e4m3", "fp16", 128, 1, 4, 64, [500], [3], scale=2.0)
    case(ev, 34, "e4m3", "bf16", 128, 1, 4, 64, [500], [3], scale=1e-6)


def test_strides_and_bounds(ev):
    """Rows of a fused projection; a table wider than needed; a max_len that is far too small or large only splits differently."""
    for max_len in (None, 1, 100000):
        case(ev, 35, "e4m3", "bf16", 128, 2, 2, 64, [333, 100], [5, 2], stride=2 * 2 * 128 + 256, max_len=max_len, extra_width=3)


def test_stale_bytes_behind_the_last_token(ev):
    """A cache of nothing but NaN, written by kv_write: what lies behind a sequence's last token does not count."""
    import torch
    rng = np.random.default_rng(36)
    for kind in ("e4m3", "int8"):
        for n in (1, 20, 33, 95):
            c = ref.Cache(5, 32, 1, 64, kind)
            table = np.array([[4, 1, 2]])
            x = torch.from_numpy(rng.standard_normal((2, n, 1, 64))).to(torch.bfloat16)
            g = to_gpu(ev, c)
            d = x.cuda()
            ev.kv_write(g, d[0], d[1], i32(table), i32([0]), i32([0, n]), n)
            c.write(x[0].float().numpy(), x[1].float().numpy(), table, [0], [0, n])
            q = torch.from_numpy(rng.standard_normal((1, 2, 64))).to(torch.bfloat16)
            out, lse = ev.kv_attention(q.cuda(), g, i32(table), i32([n]), i32([0, 1]), 1)
            want = ref.attention(c, q.double().numpy(), table, [n], [0, 1], 2, None, 0.125)
            check(out.double().cpu().numpy(), lse.double().cpu().numpy(), c, *want, 64.0, n, "bf16")


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("part", ["k", "v"])
def test_nan_reaches_only_rows_that_see_it(ev, kind, part):
    """A NaN in K or V of one tree node: siblings' outputs are those without it."""
    import torch
    rng = np.random.default_rng(37)
    n, ctx, group, dim = 8, 40, 2, 64
    kv = torch.from_numpy(rng.standard_normal((2, ctx + n, 1, dim))).to(torch.bfloat16)
    q = torch.from_numpy(rng.standard_normal((n, group, dim))).to(torch.bfloat16).cuda()
    bits = [1, 3, 5, 9, 19, 37, 67, 133]                       # node 4 is seen by itself alone
    at, start, off = i32([[0, 1]]), i32([0]), i32([0, n])
    got = []
    for bad in (False, True):
        x = kv.clone()
        if bad:
            x[0 if part == "k" else 1, ctx + 4, 0, 9] = float("nan")
        c = ev.KVCache(2, 32, 1, dim, kind)
        d = x.cuda()
        ev.kv_write(c, d[0], d[1], at, start, i32([0, ctx + n]), ctx + n)
        got.append(ev.kv_attention(q, c, at, i32([ctx + n]), off, n, tree=as_words(bits)))
    others = [0, 1, 2, 3, 5, 6, 7]
    assert torch.equal(got[0][0][others], got[1][0][others]) and torch.equal(got[0][1][others], got[1][1][others])
    bad = torch.isnan(got[1][0][4])
    if part == "k":
        assert bad.all() and torch.isnan(got[1][1][4]).all()
    else:
        assert bad[:, 9].all() and bad.sum() == group
        assert torch.equal(got[0][0][4][~bad], got[1][0][4][~bad]) and torch.equal(got[0][1][4], got[1][1][4])


def test_pages_that_are_not_there(ev):
    """Tokens of entries out of range are left out."""
    import torch
    rng = np.random.default_rng(38)
    for bad in (-1, 4, 2 ** 31 - 1, -2 ** 31):
        c = ref.Cache(4, 32, 2, 64, "e4m3", rng)
        table = np.array([[0, bad, 2], [bad, bad, bad]])
        q = torch.from_numpy(rng.standard_normal((2, 4, 64))).to(torch.bfloat16)
        out, lse = ev.kv_attention(q.cuda(), to_gpu(ev, c), i32(table), i32([96, 50]), i32([0, 1, 2]), 1)
        want = ref.attention(c, q.double().numpy(), table, [96, 50], [0, 1, 2], 2, None, 0.125)
        assert np.isneginf(want[1][1]).all()
        check(out.double().cpu().numpy(), lse.double().cpu().numpy(), c, *want, 200.0, 96, "bf16")
    # a length past the table, and a negative one
    c = ref.Cache(4, 32, 2, 64, "e4m3", rng)
    table = np.array([[0, 1], [2, 3]])
    out, lse = ev.kv_attention(q.cuda(), to_gpu(ev, c), i32(table), i32([1000, -3]), i32([0, 1, 2]), 1)
    want = ref.attention(c, q.double().numpy(), table, [1000, -3], [0, 1, 2], 2, None, 0.125)
    check(out.double().cpu().numpy(), lse.double().cpu().numpy(), c, *want, 200.0, 96, "bf16")


def test_pages_that_are_not_there_read_nothing_else(ev):
    """Whatever page 0 holds, codes and scales of NaN among it: a page that is not there has no share in the result."""
    import torch
    rng = np.random.default_rng(43)
    for kind in ("e4m3", "int8"):
        c = ref.Cache(4, 32, 2, 64, kind, rng)
        table = np.array([[2, -1, 3]])
        q = torch.from_numpy(rng.standard_normal((3, 4, 64))).to(torch.bfloat16)
        want = ref.attention(c, q.double().numpy(), table, [90], [0, 3], 2, None, 0.125)
        for scale in (np.nan, -np.nan, np.inf, 0.0, -1.0):
            c.data[0] = 0x7F if kind == "e4m3" else 0x80
            c.scales[0] = scale
            out, lse = ev.kv_attention(q.cuda(), to_gpu(ev, c), i32(table), i32([90]), i32([0, 3]), 3)
            check(out.double().cpu().numpy(), lse.double().cpu().numpy(), c, *want, 200.0, 96, "bf16")


def test_trees_larger_than_their_sequence(ev):
    """Rows whose tokens lie before the first one: their nodes are not in the cache."""
    case(ev, 44, "e4m3", "bf16", 64, 1, 2, 32, [10, 3, 40], [12, 9, 20], tree=True)


def test_rows_past_max_rows_stay(ev):
    import torch
    rng = np.random.default_rng(39)
    c = ref.Cache(3, 64, 1, 64, "e4m3", rng)
    table = np.array([[0, 1]])
    q = torch.from_numpy(rng.standard_normal((10, 1, 64))).to(torch.bfloat16)
    for max_len in (None, 100000):
        out = torch.full((10, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        ev.kv_attention(q.cuda(), to_gpu(ev, c), i32(table), i32([100]), i32([0, 10]), 4, max_len=max_len, out=out)
        want = ref.attention(c, q.double().numpy(), table, [100], [0, 10], 1, None, 0.125)
        got = out.double().cpu().numpy()
        assert (got[4:] == 7.0).all() and np.allclose(got[:4], want[0][:4], atol=0.05)


def test_same_bits_every_time(ev):
    a = case(ev, 40, "e4m3", "bf16", 128, 2, 4, 64, [2000, 50], [2, 2])
    b = case(ev, 40, "e4m3", "bf16", 128, 2, 4, 64, [2000, 50], [2, 2])
    import torch
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_graph_replays_follow_the_lengths(ev):
    """Captured once; lengths, tables and queries are read at every replay."""
    import torch
    rng = np.random.default_rng(41)
    c = ref.Cache(20, 64, 2, 64, "e4m3", rng)
    g = to_gpu(ev, c)
    table = i32(rng.permutation(20).reshape(2, 10))
    lens, off = i32([600, 20]), i32([0, 1, 2])
    q = torch.randn(2, 8, 64, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    ws = torch.empty(max(1, ev.kv_attention_workspace_bytes(g, 4, 2, 2, 1, 640)), dtype=torch.uint8, device="cuda")
    call = lambda: ev.kv_attention(q, g, table, lens, off, 1, max_len=640, out=out, out_lse=lse, workspace=ws)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a, b in ((600, 20), (3, 640), (0, 1)):
        lens.copy_(i32([a, b]))
        q.copy_(torch.randn(2, 8, 64, device="cuda").to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        eager = ev.kv_attention(q, g, table, lens, off, 1, max_len=640)
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])


def test_wrapper_refusals(ev):
    import torch
    c = ev.KVCache(4, 32, 2, 64)
    t, n, o = i32([[0, 1]]), i32([5]), i32([0, 3])
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q[:, :3]), dict(q=q.float()), dict(q=q[0]), dict(tree=torch.zeros(2, dtype=torch.int64, device="cuda")),
                dict(tree=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(lens=i32([1, 2])), dict(out=q[:2]),
                dict(out_lse=torch.zeros(3, 2, device="cuda"))):
        kw = {k: v for k, v in bad.items() if k in ("tree", "out", "out_lse")}
        with pytest.raises((TypeError, ValueError)):
            ev.kv_attention(bad.get("q", q), c, t, bad.get("lens", n), o, 3, **kw)
    with pytest.raises(ev.EvospecError) as e:
        ev.kv_attention(q, c, t, n, o, 3, scale=-1.0)
    assert e.value.status == 2


def test_workspace_refusals(ev):
    """Scratch that is not bytes on the GPU."""
    import torch
    c = ev.KVCache(4, 32, 2, 64)
    t, n, o = i32([[0, 1]]), i32([5]), i32([0, 3])
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    need = max(ev.kv_attention_workspace_bytes(c, 2, 1, 3, 3, 64), 1024)
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(need, device="cuda"), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises((TypeError, ValueError)):
            ev.kv_attention(q, c, t, n, o, 3, workspace=bad)


def test_pages_past_32_bits(ev):
    """Pages behind the first 4 GiB of a cache: the same bits as from a cache of these pages alone."""
    import torch
    rng = np.random.default_rng(45)
    heads, dim, page, pages, T = 8, 256, 256, 4500, 600          # 1 MiB a page
    far, near = ev.KVCache(pages, page, heads, dim), ev.KVCache(3, page, heads, dim)
    k, v = (torch.from_numpy(rng.standard_normal((T, heads, dim))).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((5, heads, dim))).to(torch.bfloat16).cuda()
    got = []
    for c, table in ((far, [[pages - 1, 4200, 4400]]), (near, [[2, 0, 1]])):
        ev.kv_write(c, k, v, i32(table), i32([0]), i32([0, T]), T)
        got.append(ev.kv_attention(q, c, i32(table), i32([T]), i32([0, 5]), 5))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.isfinite(got[0][0]).all()


def test_lengths_past_the_page_table(ev):
    """Lengths beyond what the page table has are cut to it."""
    import torch
    rng = np.random.default_rng(46)
    c = ref.Cache(4, 32, 2, 64, "int8", rng)
    g, table = to_gpu(ev, c), i32([[2, 0, 3]])
    q = torch.from_numpy(rng.standard_normal((3, 4, 64))).to(torch.bfloat16).cuda()
    want = ev.kv_attention(q, g, table, i32([96]), i32([0, 3]), 3)
    for n in (97, 5000, 2 ** 31 - 1):
        got = ev.kv_attention(q, g, table, i32([n]), i32([0, 3]), 3)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
